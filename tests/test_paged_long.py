"""hyq_paged_attn over long sequences, many key splits among them: outputs
within a bound relative to themselves (paged_bounds), which on the CPU is shown
to refuse outputs that are zero, too small, or lack one split's keys."""
import math

import numpy as np
import pytest

import paged_bounds as pb
import paged_common as pc
import paper_2608_27875_amd as hyq

D = 128
SCALE = 1 / math.sqrt(D)

CASES = [
    # slots before, new, Hq, Hkv, page, format, key splits, float32 additions in a row
    (32749, 1, 8, 2, 64, "bf16", 128, 300),
    (20011, 3, 10, 2, 16, "bf16", 79, 300),
    (131071, 1, 8, 1, 64, "bf16", 256, 400),
    (70003, 2, 4, 1, 16, "bf16", 256, 400),
    (65535, 1, 8, 2, 32, "int8", 256, 400),
    (131000, 2, 5, 1, 128, "fp8", 256, 400),
    (9000, 777, 8, 2, 128, "bf16", 9, 1200),
    (40001, 130, 5, 1, 256, "bf16", 64, 800),
    (0, 1500, 4, 1, 32, "bf16", 3, 600),
    (30011, 100, 8, 1, 64, "fp8", 59, 800),
]


def inputs(case, device):
    """q, page pools of values, scales and codes, the table, and k, v [Hkv, N, D]."""
    import torch
    len0, new, Hq, Hkv, page, fmt, *_ = case
    gen = torch.Generator(device=device).manual_seed(len0 + new)
    N = len0 + new
    pages = -(-N // page)
    perm = torch.randperm(pages + 2, generator=gen, device=device)[:pages]
    pool, vals = {}, {}
    for n in "kv":
        x = torch.randn((pages + 2, Hkv, page, D), generator=gen, device=device).bfloat16()
        if fmt == "bf16":
            pool[n] = x
        else:
            top = 127.0 if fmt == "int8" else 448.0
            s = x.float().abs().amax(-1) / top
            y = (x.float() / s[..., None]).clamp(-top, top)
            c = y.round().to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)
            x = c.double() * s[..., None].double() if fmt == "int8" else c.float().double() * s[..., None].double()
            pool[n], pool[n + "_scale"] = c.view(torch.uint8), s
        vals[n] = x[perm].transpose(0, 1).reshape(Hkv, -1, D)[:, :N]
    q = torch.randn((new, Hq, D), generator=gen, device=device).bfloat16()
    return q, pool, perm.to(torch.int32), vals["k"], vals["v"]


def plain(q, k, v, len0, dropped=slice(0, 0)):
    """float64 attention and masses; keys of `dropped` take no part."""
    import torch
    n, Hq, _ = q.shape
    g, N = Hq // k.shape[0], k.shape[1]
    out = torch.empty((n, Hq, D), dtype=torch.float64, device=q.device)
    mass = torch.zeros((k.shape[0], N), dtype=torch.float64, device=q.device)
    hidden = torch.arange(N, device=q.device) > len0 + torch.arange(n, device=q.device)[:, None]
    hidden[:, dropped] = True
    for h in range(Hq):
        z = (q[:, h].double() @ k[h // g].double().T.contiguous()) * SCALE
        w = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
        out[:, h] = w @ v[h // g].double()
        mass[h // g] += w.sum(0)
    return out, mass


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_outputs_and_masses(case):
    import torch
    len0, new, Hq, Hkv, page, fmt, _, sums = case
    q, pool, perm, k, v = inputs(case, torch.device("cuda"))
    mass = torch.zeros(pool["k"].shape[:3], device="cuda")
    bits, kind = pc.FORMATS[fmt]
    cache = hyq.PagedCache(Hq=Hq, Hkv=Hkv, page=page, n_pages=pool["k"].shape[0], device=q.device,
                           bits_kv=bits, kv_format=kind, bufs=dict(pool, mass=mass))
    batch = pc.batch_of([0, new], [len0], perm.cpu().numpy()[None])
    out = torch.empty((new, Hq, D), device="cuda")
    hyq.hyq_paged_attn(cache, batch, q, out, mass=hyq.MASS_ADD, ws=pc.workspace(cache, batch, True, new))
    want, wm = plain(q, k, v, len0)
    assert pb.outputs_agree(out, want, pb.relative_bound(q, k, SCALE, new * Hq // Hkv, sums))
    got = mass[perm.long()].transpose(0, 1).reshape(Hkv, -1)
    e = pb.logit_error(q, k, SCALE)
    np.testing.assert_allclose(pc.host(got[:, :len0 + new]), wm.cpu().numpy(), rtol=2 * e + (sums + 64) * 2.0 ** -24)
    assert torch.all(got[:, len0 + new:] == 0)


@pytest.mark.parametrize("case", [c for c in CASES if c[1] < 200 or c[0] == 0], ids=str)
def test_the_bound_refuses_wrong_outputs(case):
    """What the GPU test would not let pass, on its own data and case by case."""
    import torch
    len0, new, Hq, Hkv, page, fmt, splits, sums = case
    q, _, _, k, v = inputs(case, torch.device("cpu"))
    q = q[-min(new, 6):]   # the last rows: they see everything
    len0 += new - q.shape[0]
    N = len0 + q.shape[0]
    want, _ = plain(q, k, v, len0)
    rel = pb.relative_bound(q, k, SCALE, new * Hq // Hkv, sums)
    g = Hq // Hkv
    kk, vv = (x.float().repeat_interleave(g, 0) for x in (k, v))
    hidden = torch.arange(N) > len0 + torch.arange(q.shape[0])[:, None]
    z = torch.matmul(q.float().transpose(0, 1), kk.transpose(1, 2).contiguous()) * SCALE
    plain32 = torch.matmul(torch.softmax(z.masked_fill(hidden, -math.inf), -1), vv).transpose(0, 1)
    assert pb.outputs_agree(plain32, want, rel)
    assert not pb.outputs_agree(torch.zeros_like(want), want, rel)
    assert not pb.outputs_agree(want * 0.5, want, rel)
    one = want.clone()
    one[-1, 0] = 0
    assert not pb.outputs_agree(one, want, rel)
    for s in (0, splits // 2, splits - 1):
        lost, _ = plain(q, k, v, len0, slice(s * N // splits, (s + 1) * N // splits))
        assert not pb.outputs_agree(lost, want, rel), (s, splits)
