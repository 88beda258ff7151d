"""The paged serving operators: what is measured of them, and their plain forms.

A case is a dict of plain values; its ``op`` names the call:

  norm_rope  hyq.hyq_norm_rope: per-head RMS norms of q and k and the position rotation, from
             token-major projections to the [B, H, L, D] tensors of the prefill and decode calls;
  append     hyq.hyq_paged_append: the same pass for the new tokens of a ragged batch, keys and
             values into their pages (bf16, or 8-bit codes with a scale per row);
  attn       hyq.hyq_paged_attn: causal attention of each sequence's new tokens over its pages,
             and, with ``mass``, the attention weight every cached key received;
  evict      hyq.hyq_evict: the recent slots and the heaviest others of every KV head into new
             pages.

With ``own`` false, ``run`` computes the same from elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
DEV = "cuda"
EPS = 1e-6
CODE_MAX = {"int8": 127.0, "fp8": 448.0}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _norm_rope(name, B, Hq, Hkv, L, pos0=0, rot=128, interleaved=False, norm=True, packed=True):
    return dict(name=name, op="norm_rope", B=B, Hq=Hq, Hkv=Hkv, L=L, pos0=pos0, rot=rot,
                interleaved=interleaved, norm=norm, packed=packed)


def _paged(name, op, B, Hq, Hkv, length, new, page, fmt, **more):
    return dict(name=name, op=op, B=B, Hq=Hq, Hkv=Hkv, length=length, new=new, page=page, fmt=fmt,
                **more)


def _attn(name, B, Hq, Hkv, length, new, page, fmt, mass="none", mixed=False):
    return _paged(name, "attn", B, Hq, Hkv, length, new, page, fmt, mass=mass, mixed=mixed)


def _evict(name, B, Hkv, length, budget, recent, page, fmt):
    return dict(name=name, op="evict", B=B, Hkv=Hkv, length=length, budget=budget, recent=recent,
                page=page, fmt=fmt)


def listed():
    return [
        # a decode step of 16 sequences before hyq_decode_append and hyq_decode_attn: latency
        _norm_rope("norm_rope_decode_b16", 16, 32, 8, 1, pos0=32768),
        # the 8k prompt before hyq_prefill
        _norm_rope("norm_rope_8k", 1, 32, 8, 8192),
        # the batched prompt of 40 heads, odd length, interleaved pairs on half of the channels
        _norm_rope("norm_rope_b4_16k", 4, 40, 8, 16379, rot=64, interleaved=True, norm=False),
        # a step of a ragged batch of prompt chunks and single tokens into 8-bit pages
        _paged("append_ragged_fp8", "append", 9, 32, 8, 5000, 700, 16, "fp8", mixed=True),
        # a token of a short conversation: latency
        _attn("attn_decode_1k", 1, 32, 8, 1000, 1, 16, "bf16"),
        # a token of 16 long conversations served together, weights collected for the eviction
        _attn("attn_decode_b16_32k_mass", 16, 32, 8, 32768, 1, 64, "bf16", mass="add"),
        # a token of 32 conversations in 8-bit pages, groups of 5
        _attn("attn_decode_b32_8k_fp8", 32, 40, 8, 8192, 1, 32, "fp8"),
        # three drafted tokens to be verified
        _attn("attn_verify_b4_9k", 4, 32, 8, 9001, 4, 128, "bf16"),
        # the last chunk of a 32k prompt as observation window of an eviction
        _attn("attn_chunk_512_32k_mass", 1, 32, 8, 32256, 512, 64, "bf16", mass="set"),
        # a step of prompt chunks of several sequences in 8-bit pages
        _attn("attn_chunk_b3_2k_int8", 3, 40, 8, 6011, 2048, 32, "int8"),
        # a 32k prompt shrunk to 2k slots a head
        _evict("evict_32k_to_2k", 1, 8, 32768, 2048, 128, 64, "bf16"),
        # 16 conversations back to their budget
        _evict("evict_b16_8k_to_1000_fp8", 16, 8, 8192, 1000, 200, 32, "fp8"),
    ]


HEADS = [(1, 1), (4, 4), (4, 1), (8, 1), (16, 16), (12, 4), (32, 8), (32, 8), (40, 8)]
MAX_FLOPS = 0.65e12          # below the largest listed chunk
MAX_ROWS = 16 * 32768 * 8    # cached rows (batch x KV heads x slots)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope", "append", "attn", "attn", "attn", "attn", "evict"])
    while True:
        Hq, Hkv = rng.choice(HEADS)
        page = rng.choice([16, 32, 64, 128, 256])
        fmt = rng.choice(["bf16", "bf16", "int8", "fp8"])
        if op == "norm_rope":
            c = dict(op=op, B=rng.choice([1, 1, 2, 3, 16]), Hq=Hq, Hkv=Hkv,
                     L=rng.choice([1, _log_int(rng, 2, 16384), _log_int(rng, 2, 16384)]),
                     pos0=rng.choice([0, 0, _log_int(rng, 1, 1 << 20)]),
                     rot=rng.choice([128, 128, 64, 32]), interleaved=rng.random() < 0.3,
                     norm=rng.random() < 0.7, packed=rng.random() < 0.6)
            if c["B"] * c["L"] * (Hq + 2 * Hkv) > 4 * 16379 * 56:
                continue
            return c
        B = rng.choice([1, 1, 2, 3, 4, 8, 16, 32])
        length = _log_int(rng, 1, 32768) - 1
        if op == "append":
            new = rng.choice([1, _log_int(rng, 2, 1024)])
            c = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, length=length, new=new, page=page, fmt=fmt,
                     mixed=rng.random() < 0.5)
            if B * new > 16384 or B * Hkv * length > MAX_ROWS // 4:
                continue
            return c
        if op == "evict":
            length = max(length, 40)
            budget = min(length, _log_int(rng, 16, 4096))
            c = dict(op=op, B=B, Hkv=Hkv, length=length, budget=budget,
                     recent=rng.randrange(0, budget // 2 + 1), page=page, fmt=fmt)
            if B * Hkv * length > MAX_ROWS // 4:
                continue
            return c
        new = rng.choice([1, 1, 1, rng.randrange(2, 6), _log_int(rng, 6, 2048)])
        c = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, length=length, new=new, page=page, fmt=fmt,
                 mass=rng.choice(["none", "none", "set", "add"]), mixed=rng.random() < 0.3)
        if work(c)["flops"] > MAX_FLOPS or B * Hkv * (length + new) > MAX_ROWS or \
                B * Hq * new * (length + new) > 2.6e9:
            continue
        return c


def _lens(c):
    """Cached slots of every sequence: the first has the full length, the others down to half."""
    B = c["B"]
    return [c["length"] - c["length"] * b // (2 * B) for b in range(B)]


def _news(c):
    """New tokens of every sequence: mixed batches hold single tokens between the chunks, others
    shrink to three quarters (single-token batches have one each)."""
    B, n = c["B"], c["new"]
    if c["mixed"]:
        return [n if b % 3 == 0 else 1 for b in range(B)]
    return [n - n * b // (4 * B) for b in range(B)]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device=DEV, dtype=dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _projections(c, gen, T):
    """q, k, v as a projection leaves them: one packed row per token, or three tensors."""
    Hq, Hkv = c["Hq"], c["Hkv"]
    qkv = _normal(gen, T, Hq + 2 * Hkv, D)
    # heads of different sizes, and the channels that stand out in keys
    qkv[:, :Hq + Hkv] *= torch.exp2(_normal(gen, Hq + Hkv, 1))
    qkv[:, Hq:Hq + Hkv, [3, 47, 85, 122]] *= 10
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=1)
    return (q, k, v) if c.get("packed", True) else (q.contiguous(), k.contiguous(), v.contiguous())


def _rope_inputs(c, gen):
    rot = c.get("rot", D)
    w = [None, None]
    if c.get("norm", True):
        w = [(1 + 0.2 * _normal(gen, D, dtype=torch.float32)).bfloat16() for _ in range(2)]
    f = torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot
    return dict(rot=rot, interleaved=c.get("interleaved", False), q_weight=w[0], k_weight=w[1],
                inv_freq=torch.pow(1e6, -f).float())


def _tables(c, gen, lens, spare):
    """Block tables over a shuffled pool: page 0 is the null page of unused entries, then `spare`
    pages that nobody uses, then those of the sequences.  (table, pages in the pool)"""
    B, page = c["B"], c["page"]
    used = [-(-n // page) for n in lens]
    width = max(1, max(used))
    perm = torch.randperm(sum(used), generator=gen, device=DEV).to(torch.int32) + 1 + spare
    at = torch.arange(width, device=DEV)
    n = torch.tensor(used, device=DEV)
    first = (n.cumsum(0) - n).unsqueeze(1)
    table = torch.where(at < n.unsqueeze(1), perm[(first + at).clamp(max=max(0, sum(used) - 1))]
                        if sum(used) else at.to(torch.int32), 0)
    return table.to(torch.int32).contiguous(), 1 + spare + sum(used)


def _pool(c, gen, n_pages):
    """K and V pages with rows in every slot (those behind a sequence are of an earlier one)."""
    shape = (n_pages, c["Hkv"], c["page"], D)
    k, v = _normal(gen, *shape), _normal(gen, *shape)
    k[..., [3, 47, 85, 122]] *= 10
    if c["fmt"] == "bf16":
        return dict(k=k, v=v, k_scale=None, v_scale=None)
    (kc, ks), (vc, vs) = _quantized(k.float(), c["fmt"]), _quantized(v.float(), c["fmt"])
    return dict(k=kc, v=vc, k_scale=ks, v_scale=vs)


def prepare(case, seed):
    c, gen = case, _generator(seed)
    s = dict(case=c)
    if c["op"] == "norm_rope":
        B, L, Hq, Hkv = c["B"], c["L"], c["Hq"], c["Hkv"]
        s["q"], s["k"], s["v"] = _projections(c, gen, B * L)
        s.update(_rope_inputs(c, gen))
        s["pos"] = (torch.arange(L, device=DEV, dtype=torch.int32) + c["pos0"]).repeat(B)
        s["out"] = [torch.empty((B, h, L, D), dtype=torch.bfloat16, device=DEV)
                    for h in (Hq, Hkv, Hkv)]
        if own:
            import paper_2608_27875_amd as hyq
            s["shape"] = hyq.Shape(B=B, Hq=Hq, Hkv=Hkv, L=L)
            s["rope"] = _handle_rope(hyq, s)
        return s
    lens = _lens(c)
    if c["op"] == "evict":
        s["lens"] = _int32(lens)
        new_pages = -(-c["budget"] // c["page"])
        s["table"], n_pages = _tables(c, gen, lens, c["B"] * new_pages)
        s["new_table"] = (1 + torch.randperm(c["B"] * new_pages, generator=gen, device=DEV)) \
            .to(torch.int32).view(c["B"], new_pages)
        s.update(_pool(c, gen, n_pages))
        # accumulated softmax weights: a few keys hold most of it
        s["mass"] = torch.exp(2.5 * _normal(gen, n_pages, c["Hkv"], c["page"], dtype=torch.float32))
        s["keep"] = torch.empty((c["B"], c["Hkv"], c["budget"]), dtype=torch.int32, device=DEV)
        s["new_lens"] = torch.empty(c["B"], dtype=torch.int32, device=DEV)
        if own:
            import paper_2608_27875_amd as hyq
            s["cache"] = _handle_cache(hyq, c, s, c["Hkv"])
        return s
    news = _news(c)
    T = sum(news)
    s["lens"] = _int32(lens)
    s["cu_new"] = _int32([sum(news[:b]) for b in range(c["B"] + 1)])
    s["max_new"], s["max_len"] = max(news), max(lens)
    s["table"], n_pages = _tables(c, gen, [a + b for a, b in zip(lens, news)], 0)
    s.update(_pool(c, gen, n_pages))
    s["q_out"] = torch.empty((T, c["Hq"], D), dtype=torch.bfloat16, device=DEV)
    s["mass"] = None
    if c["op"] == "append":
        s["q"], s["k_new"], s["v_new"] = _projections(c, gen, T)
        s.update(_rope_inputs(c, gen))
        s["pos"] = torch.cat([torch.arange(a, a + n, device=DEV, dtype=torch.int32)
                              for a, n in zip(lens, news)])
    else:
        s["q"] = _normal(gen, T, c["Hq"], D)
        if c["mass"] != "none":
            s["mass0"] = torch.rand((n_pages, c["Hkv"], c["page"]), generator=gen, device=DEV)
            s["mass"] = s["mass0"].clone()
    if own:
        import paper_2608_27875_amd as hyq
        s["cache"] = _handle_cache(hyq, c, s, c["Hq"])
        s["batch"] = hyq.PagedBatch(cu_new=s["cu_new"], lens=s["lens"], table=s["table"],
                                    max_new=s["max_new"], max_len=s["max_len"])
        if c["op"] == "append":
            s["rope"] = _handle_rope(hyq, s)
        else:
            s["ws"] = torch.empty(hyq.hyq_paged_ws_bytes(s["cache"], s["batch"], c["mass"] != "none"),
                                  dtype=torch.uint8, device=DEV)
    return s


def _handle_rope(hyq, s):
    return hyq.Rope(rot_dim=s["rot"], interleaved=s["interleaved"], eps=EPS,
                    q_weight=s["q_weight"], k_weight=s["k_weight"], inv_freq=s["inv_freq"])


def _handle_cache(hyq, c, s, Hq):
    bits, fmt = {"bf16": (16, hyq.FMT_INT), "int8": (8, hyq.FMT_INT), "fp8": (8, hyq.FMT_FP8)}[c["fmt"]]
    bufs = {n: s[n] for n in ("k", "v", "k_scale", "v_scale", "mass")}
    return hyq.PagedCache(Hq=Hq, Hkv=c["Hkv"], page=c["page"], n_pages=s["k"].shape[0],
                          device=s["k"].device, bits_kv=bits, kv_format=fmt, bufs=bufs)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if c["op"] == "norm_rope":
        if own:
            import paper_2608_27875_amd as hyq
            hyq.hyq_norm_rope(s["shape"], s["rope"], s["q"], s["k"], s["v"], s["pos"], *s["out"])
            return s["out"]
        B, L = c["B"], c["L"]
        rows = [_normed_rotated(s, s["q"], s["q_weight"]), _normed_rotated(s, s["k"], s["k_weight"]),
                s["v"]]
        return [x.view(B, L, -1, D).transpose(1, 2).bfloat16().contiguous() for x in rows]
    if c["op"] == "append":
        if own:
            import paper_2608_27875_amd as hyq
            hyq.hyq_paged_append(s["cache"], s["batch"], s["rope"], s["q"], s["k_new"], s["v_new"],
                                 s["pos"], s["q_out"])
        else:
            _plain_append(c, s)
        return dict(q=s["q_out"], **_values(c, s["k"], s["k_scale"], s["v"], s["v_scale"]))
    if c["op"] == "attn":
        if c["mass"] == "add":
            s["mass"].copy_(s["mass0"])   # every pass adds to the same weights
        if own:
            import paper_2608_27875_amd as hyq
            mode = {"none": hyq.MASS_NONE, "add": hyq.MASS_ADD, "set": hyq.MASS_SET}[c["mass"]]
            hyq.hyq_paged_attn(s["cache"], s["batch"], s["q"], s["q_out"], out_dtype=1, mass=mode,
                               ws=s["ws"])
        else:
            _plain_attention(c, s)
        return dict(out=s["q_out"]) if c["mass"] == "none" else dict(out=s["q_out"], mass=s["mass"])
    if own:
        import paper_2608_27875_amd as hyq
        hyq.hyq_evict(s["cache"], s["lens"], s["table"], s["new_table"], s["keep"], s["new_lens"],
                      max_len=c["length"], budget=c["budget"], recent=c["recent"])
    else:
        _plain_evict(c, s)
    n = 1 + s["new_table"].numel()   # the pages that the kept rows went to
    r = dict(keep=s["keep"], new_lens=s["new_lens"], mass=s["mass"][1:n])
    if c["fmt"] == "bf16":
        return dict(r, k=s["k"][1:n], v=s["v"][1:n])
    return dict(r, **_values(c, s["k"][1:n], s["k_scale"][1:n], s["v"][1:n], s["v_scale"][1:n]))


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _quantized(x, fmt):
    """Rows of x (float32) as (codes, scales): s = max|x| / c per row, code nearest to x / s."""
    s = x.abs().amax(dim=-1) / CODE_MAX[fmt]
    y = torch.where(s.unsqueeze(-1) > 0, x / s.unsqueeze(-1), 0.0)
    if fmt == "fp8":
        return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), s
    return y.round().clamp(-127, 127).to(torch.int8).view(torch.uint8), s


def _decoded(fmt, codes, scale):
    """Pages as float32 values."""
    if fmt == "bf16":
        return codes.float()
    typed = codes.view(torch.float8_e4m3fn if fmt == "fp8" else torch.int8)
    return typed.float() * scale.unsqueeze(-1)


def _values(c, k, k_scale, v, v_scale):
    """What the pages hold: bf16 rows, E4M3 numbers and their scales, int8 codes as the values
    they stand for."""
    if c["fmt"] == "bf16":
        return dict(k=k, v=v)
    if c["fmt"] == "fp8":
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    else:
        k, v = _decoded("int8", k, k_scale).bfloat16(), _decoded("int8", v, v_scale).bfloat16()
    return dict(k=k, k_scale=k_scale, v=v, v_scale=v_scale)


def _normed_rotated(s, x, weight):
    """Rows x [T, H, D]: RMS norm (where there are weights), then the rotation, in float32."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight.float()
    rot = s["rot"]
    angle = s["pos"].double().unsqueeze(1) * s["inv_freq"].double()   # far positions need 64 bits
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    r = x[..., :rot]
    if s["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([r, x[..., rot:]], dim=-1)


def _token_places(s, T):
    """Sequence and index within it of every new token."""
    t = torch.arange(T, device=DEV)
    seq = torch.searchsorted(s["cu_new"][1:].long(), t, right=True)
    return seq, t - s["cu_new"][seq]


def _plain_append(c, s):
    T, page = s["q"].shape[0], c["page"]
    s["q_out"].copy_(_normed_rotated(s, s["q"], s["q_weight"]))
    seq, i = _token_places(s, T)
    slot = s["lens"][seq] + i
    p, off = s["table"][seq, slot // page].long(), slot % page
    for_k, for_v = _normed_rotated(s, s["k_new"], s["k_weight"]), s["v_new"].float()
    if c["fmt"] == "bf16":
        s["k"][p, :, off] = for_k.bfloat16()
        s["v"][p, :, off] = for_v.bfloat16()
        return
    s["k"][p, :, off], s["k_scale"][p, :, off] = _quantized(for_k, c["fmt"])
    s["v"][p, :, off], s["v_scale"][p, :, off] = _quantized(for_v, c["fmt"])


def _by_slot(pool, table):
    """Pages in the order of the table: [B, Hkv, slots, ...]."""
    x = pool[table.long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], x.shape[2] * x.shape[3], *x.shape[4:])


def _plain_attention(c, s):
    B, Hkv, g, n = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], s["max_new"]
    T, page = s["q"].shape[0], c["page"]
    K = _decoded(c["fmt"], _by_slot(s["k"], s["table"]),
                 None if s["k_scale"] is None else _by_slot(s["k_scale"], s["table"]))
    V = _decoded(c["fmt"], _by_slot(s["v"], s["table"]),
                 None if s["v_scale"] is None else _by_slot(s["v_scale"], s["table"]))
    N = K.shape[2]
    i = torch.arange(n, device=DEV)
    rows = (s["cu_new"][:B, None] + i).clamp(max=T - 1).long()
    q = s["q"].float()[rows].view(B, n, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * g, D)
    z = torch.matmul(q, K.transpose(-1, -2).contiguous()) / math.sqrt(D)
    slot = torch.arange(N, device=DEV)
    there = i < (s["cu_new"][1:] - s["cu_new"][:B]).unsqueeze(1)                   # [B, n]
    seen = (slot < (s["lens"][:, None] + i + 1).unsqueeze(2)) & there.unsqueeze(2)   # [B, n, N]
    z = z.view(B, Hkv, n, g, N).masked_fill_(~seen[:, None, :, None], -math.inf).view(B, Hkv, n * g, N)
    top = z.amax(dim=-1, keepdim=True)
    z = z.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    z = z.div_(z.sum(dim=-1, keepdim=True).clamp_min(1e-30))
    o = torch.matmul(z, V).view(B, Hkv, n, g, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hkv * g, D)
    seq, at = _token_places(s, T)
    s["q_out"].copy_(o[seq, at])
    if c["mass"] == "none":
        return
    got = z.sum(dim=2)                                                            # [B, Hkv, N]
    total = s["lens"] + s["cu_new"][1:] - s["cu_new"][:B]
    p, off = s["table"].long()[:, slot // page], (slot % page).expand(B, N)
    old = s["mass"][p, :, off]                                                    # [B, N, Hkv]
    got = got.transpose(1, 2) + old if c["mass"] == "add" else got.transpose(1, 2)
    s["mass"][p, :, off] = torch.where((slot < total.unsqueeze(1)).unsqueeze(2), got, old)


def _plain_evict(c, s):
    B, Hkv, budget, page = c["B"], c["Hkv"], c["budget"], c["page"]
    m = _by_slot(s["mass"], s["table"])
    n = s["lens"].long().view(B, 1, 1)
    slot = torch.arange(m.shape[2], device=DEV)
    m = torch.where(slot < n, torch.where(slot >= n - c["recent"], math.inf, m), -math.inf)
    m = torch.nn.functional.pad(m, (0, max(0, budget - m.shape[2])), value=-math.inf)
    # the largest first, equal ones by their slot
    kept = torch.sort(m, dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = torch.sort(kept, dim=-1).values
    there = kept < n
    s["keep"].copy_(torch.where(there, kept, 0x7FFFFFFF))
    s["new_lens"].copy_(s["lens"].clamp(max=budget))
    src = kept.clamp(max=s["table"].shape[1] * page - 1)
    b = torch.arange(B, device=DEV).view(B, 1, 1)
    h = torch.arange(Hkv, device=DEV).view(1, Hkv, 1)
    at = torch.arange(budget, device=DEV)
    p, off = s["table"].long()[b, src // page], src % page
    p2, off2 = s["new_table"].long()[:, None, at // page].expand(B, Hkv, budget), (at % page).expand(B, Hkv, budget)
    h = h.expand(B, Hkv, budget)
    _moved(s["mass"], p, off, p2, off2, h, there)
    _moved(s["k"], p, off, p2, off2, h, there)
    _moved(s["v"], p, off, p2, off2, h, there)
    if c["fmt"] != "bf16":
        _moved(s["k_scale"], p, off, p2, off2, h, there)
        _moved(s["v_scale"], p, off, p2, off2, h, there)


def _moved(pool, p, off, p2, off2, h, there):
    there = there.view(there.shape + (1,) * (pool.dim() - 3))
    pool[p2, h, off2] = torch.where(there, pool[p, h, off], pool[p2, h, off2])


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _row_bytes(c):
    """Bytes of a cached key row (or value row), its scale among them."""
    return 2 * D if c["fmt"] == "bf16" else D + 4


def work(case):
    c = case
    if c["op"] == "norm_rope":
        T = c["B"] * c["L"]
        rows = T * (c["Hq"] + 2 * c["Hkv"])
        turned = T * (c["Hq"] + c["Hkv"])
        return dict(bytes=rows * D * 4 + T * 4,
                    flops=turned * (3 * c["rot"] + (4 * D if c["norm"] else 0)))
    if c["op"] == "evict":
        lens = _lens(c)
        kept = sum(min(n, c["budget"]) for n in lens)
        return dict(bytes=c["Hkv"] * (4 * sum(lens) + kept * (4 * _row_bytes(c) + 8)), flops=0)
    news, lens = _news(c), _lens(c)
    T, slots = sum(news), sum(news) + sum(lens)
    if c["op"] == "append":
        return dict(bytes=T * (c["Hq"] * D * 4 + 2 * c["Hkv"] * (2 * D + _row_bytes(c)) + 4),
                    flops=T * (c["Hq"] + c["Hkv"]) * 7 * D)
    n = slots * c["Hkv"] * 2 * _row_bytes(c) + T * c["Hq"] * D * 4
    n += {"none": 0, "set": 4, "add": 8}[c["mass"]] * slots * c["Hkv"]
    pairs = sum(a * t + t * (t + 1) // 2 for a, t in zip(lens, news))
    return dict(bytes=n, flops=4 * D * c["Hq"] * pairs)


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm_rope":
        B, L = c["B"], c["L"]
        q, k = _exact_rows(s, s["q"], s["q_weight"]), _exact_rows(s, s["k"], s["k_weight"])
        return [x.double().unflatten(0, (B, L)).movedim(2, 1).contiguous() for x in (q, k, s["v"])]
    if c["op"] == "append":
        return _exact_append(c, s)
    if c["op"] == "attn":
        return _exact_attention(c, s)
    return _exact_evict(c, s)


def _exact_rows(s, x, weight):
    """The rotation as a product of complex numbers."""
    x = x.double()
    if weight is not None:
        x = x / (x.square().sum(-1, keepdim=True) / D + EPS).sqrt() * weight.double()
    rot = s["rot"]
    turn = torch.outer(s["pos"].double(), s["inv_freq"].double())
    turn = torch.polar(torch.ones_like(turn), turn)[:, None]
    y = x.clone()
    if s["interleaved"]:
        z = torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) * turn
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    else:
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def _exact_value(fmt, codes, scale):
    if fmt == "bf16":
        return codes.double()
    if fmt == "int8":
        return codes.view(torch.int8).double() * scale.double()[..., None]
    u = codes.long()
    e, f = (u >> 3) & 15, (u & 7).double()
    size = torch.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * torch.exp2(e.double() - 7))
    return torch.where(u >= 128, -size, size) * scale.double()[..., None]


def _exact_rounded(x, fmt):
    """(the value of the code nearest to every entry, the scale of every row); E4M3 numbers are
    given without their scale, as they are returned."""
    s = x.abs().amax(-1, keepdim=True) / CODE_MAX[fmt]
    y = torch.where(s > 0, x / s, torch.zeros_like(x))
    if fmt == "int8":
        return y.round() * s, s[..., 0]
    e = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (y / step).round() * step, s[..., 0]


def _exact_pools(c, s):
    unit = torch.ones_like(s["k_scale"]) if c["fmt"] == "fp8" else s["k_scale"]
    pools = dict(k=_exact_value(c["fmt"], s["k"], unit),
                 v=_exact_value(c["fmt"], s["v"], unit if c["fmt"] == "fp8" else s["v_scale"]))
    if c["fmt"] != "bf16":
        pools.update(k_scale=s["k_scale"].double(), v_scale=s["v_scale"].double())
    return pools


def _exact_append(c, s):
    news, lens, page = _news(c), _lens(c), c["page"]
    k, v = _exact_rows(s, s["k_new"], s["k_weight"]), s["v_new"].double()
    r = dict(q=_exact_rows(s, s["q"], s["q_weight"]))
    pools = _exact_pools(c, s)
    if c["fmt"] != "bf16":
        (k, ks), (v, vs) = _exact_rounded(k, c["fmt"]), _exact_rounded(v, c["fmt"])
    place = torch.cat([torch.arange(a, a + n) for a, n in zip(lens, news)])
    whose = torch.cat([torch.full((n,), b) for b, n in enumerate(news)])
    table = s["table"].cpu()
    p, off = table[whose, place // page].long().to(DEV), (place % page).to(DEV)
    pools["k"][p, :, off], pools["v"][p, :, off] = k, v
    if c["fmt"] != "bf16":
        pools["k_scale"][p, :, off], pools["v_scale"][p, :, off] = ks, vs
    return dict(r, **pools)


def _exact_attention(c, s):
    news, lens, page = _news(c), _lens(c), c["page"]
    g, T = c["Hq"] // c["Hkv"], sum(news)
    out = torch.zeros((T, c["Hq"], D), dtype=torch.float64, device=DEV)
    mass = None if c["mass"] == "none" else s["mass"].double()
    t0 = 0
    for b, (n, t) in enumerate(zip(lens, news)):
        total = n + t
        pages = s["table"][b, :-(-total // page)].long()
        future = torch.arange(total, device=DEV) > torch.arange(n, total, device=DEV)[:, None]
        for j in range(c["Hkv"]):
            def rows(x, sc):
                y = _exact_value(c["fmt"], x[pages, j], None if sc is None else sc[pages, j])
                return y.reshape(-1, D)[:total]
            K, V = rows(s["k"], s["k_scale"]), rows(s["v"], s["v_scale"])
            got = torch.zeros(total, dtype=torch.float64, device=DEV)
            for h in range(j * g, (j + 1) * g):
                z = (s["q"][t0:t0 + t, h].double() @ K.T) / math.sqrt(D)
                w = torch.softmax(z.masked_fill(future, -math.inf), dim=-1)
                out[t0:t0 + t, h] = w @ V
                got += w.sum(0)
            if mass is not None:
                flat = mass[pages, j].reshape(-1)
                flat[:total] = got + flat[:total] if c["mass"] == "add" else got
                mass[pages, j] = flat.view(-1, page)
        t0 += t
    return dict(out=out) if mass is None else dict(out=out, mass=mass)


def _exact_evict(c, s):
    page, budget = c["page"], c["budget"]
    pools = dict(_exact_pools(c, s), mass=s["mass"].double())
    for b, n in enumerate(_lens(c)):
        old = s["table"][b].long().repeat_interleave(page)
        new = s["new_table"][b].long().repeat_interleave(page)
        for j in range(c["Hkv"]):
            at = torch.arange(n, device=DEV)
            w = s["mass"][old[:n], j, at % page].double()
            w[max(0, n - c["recent"]):] = math.inf
            kept = torch.argsort(-w, stable=True)[:budget].sort().values
            to = torch.arange(kept.numel(), device=DEV)
            for x in pools.values():
                x[new[to], j, to % page] = x[old[kept], j, kept % page]
    n = 1 + s["new_table"].numel()
    # which slots are kept is a whole number: it is compared with the plain form's alone
    return dict({k: x[1:n] for k, x in pools.items()}, keep=None, new_lens=None)
