"""Helpers of the paged serving tests: seeded batches over shuffled pages, the
same data as torch tensors and as the oracle's float64 values, and tolerances."""
from __future__ import annotations

import numpy as np

import paper_2608_27875_amd as hyq
from oracle import paged_oracle as po
from paper_2608_27875_amd import gen

D = 128
FORMATS = {"bf16": (16, hyq.FMT_INT), "int8": (8, hyq.FMT_INT), "fp8": (8, hyq.FMT_FP8)}


def bits(rng, *shape, scale=1.0):
    """bf16 bit patterns of normal values."""
    return gen.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))


def dev(x):
    import torch
    x = np.ascontiguousarray(x)
    if x.dtype == np.uint16:
        return torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).cuda()
    return torch.from_numpy(x).cuda()


def host(t):
    """float64 of a torch tensor."""
    import torch
    return t.to(torch.float64).cpu().numpy()


def tables(rng, lens, page, extra_pages=3, width=None):
    """(table, n_pages): shuffled pages; entries behind a sequence are -1, a
    large value or someone's page."""
    used = [-(-int(n) // page) for n in lens]
    n_pages = sum(used) + extra_pages
    perm = rng.permutation(n_pages)
    width = max(1, max(used), width or 0)
    table = rng.choice([-1, 1 << 30, 0], size=(len(lens), width)).astype(np.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = perm[at:at + u]
        at += u
    return table, n_pages


def pool(rng, fmt, n_pages, Hkv, page, poison=True):
    """Pages full of rows: dict of numpy buffers, and their values in float64."""
    out, vals = {}, {}
    for n in ("k", "v"):
        b = bits(rng, n_pages, Hkv, page, D)
        if n == "k":   # some channels stand out
            f = po.bf16(b)
            f[..., [3, 47, 85, 122]] *= 10
            b = gen.f32_to_bf16_bits(f.astype(np.float32))
        if fmt == "bf16":
            out[n], vals[n] = b, po.bf16(b)
        else:
            code, s, v = po.quantize_row(po.bf16(b), "int" if fmt == "int8" else "fp8")
            out[n], out[n + "_scale"], vals[n] = code.view(np.uint8), s, v
    return out, vals


def cache_of(bufs, fmt, Hq, mass=None):
    n_pages, Hkv, page, _ = bufs["k"].shape
    b, f = FORMATS[fmt]
    d = {n: dev(x) for n, x in bufs.items()}
    d["mass"] = None if mass is None else dev(mass)
    return hyq.PagedCache(Hq=Hq, Hkv=Hkv, page=page, n_pages=n_pages, device=d["k"].device,
                          bits_kv=b, kv_format=f, bufs=d)


def batch_of(cu, lens, table, max_new=None, max_len=None):
    cu, lens = np.asarray(cu, np.int32), np.asarray(lens, np.int32)
    return hyq.PagedBatch(cu_new=dev(cu), lens=dev(lens), table=dev(np.asarray(table, np.int32)),
                          max_new=int(np.diff(cu).max()) if max_new is None else max_new,
                          max_len=int(lens.max()) if max_len is None else max_len)


def workspace(cache, batch, mass, T):
    import torch
    n = hyq.hyq_paged_ws_bytes(cache, batch, mass, T)
    return torch.full((max(n, 16),), 255, dtype=torch.uint8, device=cache.device)   # NaN partials


def logit_error(qv, kv, scale, chunk=4096):
    """Bound on the error of a logit: 128 products summed in float32, and the
    scaling, relative to the sum of their magnitudes."""
    big = np.abs(qv).reshape(-1, D).max(0) @ np.abs(kv).reshape(-1, D).max(0)
    return scale * big * 130 * 2.0 ** -24


def out_tolerance(qv, vals, scale, new_rows, bf16_out):
    """(absolute, relative) tolerance of attention outputs.  A logit off by e
    moves a weight by e and the sum by e; weights enter as a high + low bf16
    pair (2^-16) up to 16 rows a KV head, as bf16 (2^-8) beyond; a bf16 output
    is off by 2^-8 of its value."""
    e = logit_error(qv, vals["k"], scale)
    w = 2.0 ** -16 if new_rows <= 16 else 2.0 ** -8
    return (2 * e + w + 2.0 ** -20) * np.abs(vals["v"]).max(), 2.0 ** -8 if bf16_out else 2.0 ** -23
