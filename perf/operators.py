"""Performance cases of the operators between a decoder's projections: rotary positions, the paged key-value cache and the
attention of one new token over it.

A case is a dict of plain values; ``kind`` says what a pass is:

  rotary   rotary positions on a [tokens, heads, head_dim] view (qii_rotary), forward or gradient
  write    keys and values of new tokens into the paged cache (qii_kv_append: rotated, rounded to the cache's type), then read
           back (qii_kv_read), as a program does whose next chunk of a prompt attends to the earlier ones
  read     a range of cached positions of every sequence as dense rows (qii_kv_read)
  attend   attention of one new token of every sequence over its cached positions (qii_paged_attention)
  step     the attention of a decoding step: the new token's key and value into the cache, then its attention, both rotated

The cache is NVFP4 (E2M1 codes, one E4M3 scale per 16 elements of a head, one f32 scale per tensor) or bf16, in pages of
``page`` positions.  A page table maps (sequence, page of the sequence) to a page, -1 where none is mapped.

Layouts: bf16 [pages, kv_heads, page, head_dim]; NVFP4 codes [pages, kv_heads, page, head_dim / 2], low nibble first; scales of
the keys [pages, kv_heads, page, head_dim / 16], of the values [pages, kv_heads, head_dim / 16, page].
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MAX_CACHE_BYTES = 3200 << 20         # of a drawn case's cache: no more than the largest listed one reads
MAX_EXPANDED = 1 << 31               # elements of all sequences' keys, each filled up to the longest one, of a drawn case
MAX_ROTARY = 32768 * 32 * 128        # elements of a drawn case


# ------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # queries of four sequences that decode together, f32: launches count
        dict(name="rotary_step_f32", kind="rotary", tokens=4, heads=16, D=128, rot=128, layout="half", scaling="none", dt="f32",
             inverse=False, seqs=4, start=1000, pad=0),
        # queries and keys of the 1.9B decoder's fused projection (row of 6144 with the values) at 32768 tokens a step
        dict(name="rotary_qk_train", kind="rotary", tokens=32768, heads=32, D=128, rot=128, layout="half", scaling="none", dt="bf16",
             inverse=False, seqs=16, start=0, pad=2048),
        # a gradient with nothing even: part of the head rotated, pairs side by side, ragged tokens, a scaled long context
        dict(name="rotary_grad_odd", kind="rotary", tokens=5003, heads=24, D=96, rot=48, layout="interleaved", scaling="by_parts",
             dt="f32", inverse=True, seqs=7, start=30000, pad=96),
        # one new token of each of 32 sequences into the cache
        dict(name="write_step", kind="write", seqs=32, new=1, past=1500, kv=8, D=128, page=16, cache="nvfp4", mode="rtn", dt="bf16",
             out="bf16", rot=128, layout="half"),
        # prompts of up to 2048 tokens, the decoder's 16 heads, the forward pass's 4/6 rounding
        dict(name="write_prompts", kind="write", seqs=12, new=2048, past=0, kv=16, D=128, page=64, cache="nvfp4", mode="rtn_46", dt="bf16",
             out="bf16", rot=128, layout="half"),
        # f32 projections, a head dimension and a page size that are no powers of two, half of the head rotated
        dict(name="write_odd", kind="write", seqs=5, new=389, past=1001, kv=5, D=80, page=48, cache="nvfp4", mode="rtn", dt="f32",
             out="f32", rot=40, layout="interleaved"),
        # cached prefixes as dense bf16 rows, for a chunk of a prompt that attends to them
        dict(name="read_prefix", kind="read", seqs=4, new=8192, past=0, kv=8, D=128, page=32, cache="nvfp4", out="bf16"),
        # the first words of an answer: two short sequences, the decoder's 16 heads, latency
        dict(name="attend_short", kind="attend", seqs=2, heads=16, kv=16, D=128, page=16, cache="bf16", dt="bf16", min_len=1, max_len=33,
             window=0, starts=False, rope=False),
        # a serving batch: 64 sequences of up to 4096 tokens, 32 query heads on 8 of keys and values, NVFP4
        dict(name="attend_batch_nvfp4", kind="attend", seqs=64, heads=32, kv=8, D=128, page=16, cache="nvfp4", dt="bf16", min_len=100,
             max_len=4096, window=0, starts=False, rope=False),
        # one sequence with a long context: few rows, the work is along the length
        dict(name="attend_long_nvfp4", kind="attend", seqs=1, heads=32, kv=8, D=128, page=64, cache="nvfp4", dt="bf16", min_len=131071,
             max_len=131071, window=0, starts=False, rope=True),
        # f32, a window, sequences that begin late or have no keys left, odd head dimension and page
        dict(name="attend_window_odd", kind="attend", seqs=13, heads=10, kv=2, D=80, page=48, cache="nvfp4", dt="f32", min_len=0,
             max_len=5001, window=1500, starts=True, rope=False),
        # the decoder's own heads (16 x 128, no sharing) with a bf16 cache: the new token written and attended to; the largest
        dict(name="step_bf16", kind="step", seqs=96, heads=16, kv=16, D=128, page=32, cache="bf16", dt="bf16", mode="rtn", min_len=500,
             max_len=8000, window=0, starts=False, rope=True),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: 1 to 32768 tokens, 1 to 128 sequences, cached lengths 1 to 131072, head dimensions 16 to 256, both caches and types."""
    kind = rng.choice(["rotary", "rotary", "write", "write", "read", "attend", "attend", "attend", "attend", "step", "step"])
    D = rng.choice([64, 128, 128, 128, 256, 16 * rng.randint(1, 16)])
    layout, page = rng.choice(["half", "interleaved"]), rng.choice([16, 16, 32, 64, 128, 16 * rng.randint(1, 12)])
    rot = rng.choice([D, D, 2 * rng.randint(1, D // 2)])
    cache, dt = rng.choice(["nvfp4", "nvfp4", "bf16"]), rng.choice(["bf16", "bf16", "f32"])
    if kind == "rotary":
        while True:
            tokens, heads = _log(rng, 1, 32768), _log(rng, 1, 64)
            if tokens * heads * D <= MAX_ROTARY:
                return dict(kind=kind, tokens=tokens, heads=heads, D=D, rot=rot, layout=layout, dt=dt, inverse=rng.random() < 0.5,
                            scaling=rng.choice(["none", "none", "linear", "base", "by_parts"]), seqs=min(tokens, _log(rng, 1, 64)),
                            start=rng.choice([0, _log(rng, 1, 100000)]), pad=rng.choice([0, D, 16 * rng.randint(0, 200)]))
    while True:
        seqs, kv = _log(rng, 1, 128), _log(rng, 1, 32)
        if kind in ("write", "read"):
            new = 1 if rng.random() < 0.3 else _log(rng, 1, 8192)
            case = dict(kind=kind, seqs=seqs, new=new, past=rng.choice([0, _log(rng, 1, 4096)]), kv=kv, D=D, page=page, cache=cache,
                        out=rng.choice(["bf16", "bf16", "f32"]))
            if kind == "write":
                case.update(mode=rng.choice(["rtn", "rtn_46"]), dt=dt, rot=rng.choice([0, rot]), layout=layout)
            if seqs * new * kv * D <= MAX_ROTARY and seqs * (new + case["past"]) * kv * D <= 8 * MAX_ROTARY:
                return case
            continue
        longest = _log(rng, 1, 131072)
        case = dict(kind=kind, seqs=seqs, heads=kv * rng.choice([1, 2, 4, 8, rng.randint(1, 24)]), kv=kv, D=D, page=page, cache=cache, dt=dt,
                    min_len=rng.choice([0 if kind == "attend" else 1, longest]), max_len=longest,
                    window=rng.choice([0, 0, _log(rng, 1, 8192)]), starts=rng.random() < 0.25, rope=rng.random() < 0.5)
        if kind == "step":
            case.update(mode="rtn", rope=True)
        expanded = seqs * longest * kv * D
        if expanded <= MAX_EXPANDED and 2 * _element_bytes(case) * expanded <= MAX_CACHE_BYTES:
            return case


# ------------------------------------------------------------------------------------------------- inputs
def _element_bytes(case):
    return 2.0 if case["cache"] == "bf16" else 0.5 + 1.0 / 16


def _lengths(case):
    """Cached lengths (the new token's among them): of the case alone, ragged between its bounds, the longest one first."""
    lo, hi, n = case["min_len"], case["max_len"], case["seqs"]
    return [hi] + [lo + (i * 2654435761 % (1 << 32)) * (hi - lo + 1) // (1 << 32) for i in range(1, n)]


def _starts(case, lengths):
    """First position that counts, where a case has them: late ones, and one past the last key."""
    return [0 if i % 3 else n // 2 + (n if i % 6 else 0) for i, n in enumerate(lengths)]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(shape, dt, g, std=1.0):
    return (torch.randn(shape, device="cuda", dtype=torch.float32, generator=g) * std).to(dt)


def _keys(shape, dt, g):
    """N(0, 1) with one element of a head in 32 four times larger, the same ones for all tokens: keys have such channels."""
    k = torch.randn(shape, device="cuda", dtype=torch.float32, generator=g)
    k[..., 5::32] *= 4.0
    return k.to(dt)


def _table(positions, rot, scaling="none", base=10000.0, factor=4.0, original=8192):
    """cos and sin of every position's angles, f32 [positions, 2, rot / 2] (times the magnitude of the scaling)."""
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    magnitude = 1.0
    if scaling == "base":
        base = base * factor ** (rot / max(rot - 2, 1))
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":      # long wavelengths interpolated, short ones kept, a ramp between 32 turns and 1 turn
        turns = original * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
        magnitude = 0.1 * math.log(factor) + 1.0
    a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * f
    return torch.stack((torch.cos(a), torch.sin(a)), dim=1).mul_(magnitude).float()


def _page_table(capacity, page, g):
    """Pages for `capacity[i]` positions of sequence i, in no order, and two spare ones; -1 beyond."""
    counts = torch.tensor([-(-c // page) for c in capacity], device="cuda")
    total, widest = int(counts.sum()), max(1, int(counts.max()))
    mapped = torch.arange(widest, device="cuda")[None, :] < counts[:, None]
    table = torch.full((len(capacity), widest), -1, dtype=torch.int32, device="cuda")
    table[mapped] = torch.randperm(total + 2, device="cuda", generator=g)[:total].to(torch.int32)
    return table, total + 2


def _empty_cache(case, pages):
    """Memory that nothing was written to yet may hold anything: here NaN (scale byte 0x7F)."""
    kv, page, D = case["kv"], case["page"], case["D"]
    if case["cache"] == "bf16":
        return {"k": torch.full((pages, kv, page, D), float("nan"), dtype=torch.bfloat16, device="cuda"),
                "v": torch.full((pages, kv, page, D), float("nan"), dtype=torch.bfloat16, device="cuda"),
                "k_scales": None, "v_scales": None, "k_scale": None, "v_scale": None}
    u8 = dict(dtype=torch.uint8, device="cuda")
    return {"k": torch.full((pages, kv, page, D // 2), 0x77, **u8), "v": torch.full((pages, kv, page, D // 2), 0x77, **u8),
            "k_scales": torch.full((pages, kv, page, D // 16), 0x7F, **u8), "v_scales": torch.full((pages, kv, D // 16, page), 0x7F, **u8),
            # maxima of about 20 and 6 under the forward pass's rule amax / (6 * 448), as a program calibrates them
            "k_scale": torch.full((1,), 20.0 / (6 * 448), device="cuda"), "v_scale": torch.full((1,), 6.0 / (6 * 448), device="cuda")}


def _tokens(case):
    """Sequence and position of every new token of a write or read: `new` of the first sequence, between one and that of the others."""
    counts = _lengths(dict(case, min_len=1, max_len=case["new"]))
    pasts = [case["past"] * (i % 4 + 1) // 4 for i in range(case["seqs"])]
    seqs = torch.cat([torch.full((c,), i) for i, c in enumerate(counts)])
    positions = torch.cat([torch.arange(p, p + c) for p, c in zip(pasts, counts)])
    return counts, pasts, seqs.to(torch.int32).cuda(), positions.to(torch.int32).cuda()


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case)
    kind, D = case["kind"], case["D"]
    if kind == "rotary":
        n, h, dt = case["tokens"], case["heads"], DTYPES[case["dt"]]
        per = -(-n // case["seqs"])
        wide = _normal((n, h * D + case["pad"]), dt, g)      # the view leaves out `pad` elements of each token (the values)
        s.update(x=wide[:, : h * D].view(n, h, D), y=torch.empty((n, h, D), dtype=dt, device="cuda"),
                 positions=(case["start"] + torch.arange(n, device="cuda") % per).to(torch.int32),
                 table=_table(case["start"] + per, case["rot"], case["scaling"]))
        return s
    kv, page = case["kv"], case["page"]
    if kind in ("write", "read"):
        counts, pasts, seqs, positions = _tokens(case)
        table, pages = _page_table([p + c for p, c in zip(pasts, counts)], page, g)
        n, out = len(positions), DTYPES[case["out"]]
        s.update(cache_buffers=_empty_cache(case, pages), page_table=table, seq_ids=seqs, positions=positions,
                 k_out=torch.empty((n, kv, D), dtype=out, device="cuda"), v_out=torch.empty((n, kv, D), dtype=out, device="cuda"))
        dt = DTYPES[case.get("dt", "bf16")]
        k, v = _keys((n, kv, D), dt, g), _normal((n, kv, D), dt, g)
        if kind == "read":
            _write(s["cache_buffers"], k.float(), v.float(), seqs, positions, table, "rtn")
        else:
            s.update(k=k, v=v, table=_table(case["past"] + case["new"], case["rot"]) if case["rot"] else None)
        return s
    h, dt, lengths = case["heads"], DTYPES[case["dt"]], _lengths(case)
    table, pages = _page_table(lengths, page, g)
    s.update(cache_buffers=_filled_cache(case, pages, lengths, table, g), page_table=table, q=_normal((case["seqs"], h, D), dt, g),
             lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), scale=D ** -0.5, layout="half",
             starts=torch.tensor(_starts(case, lengths), dtype=torch.int32, device="cuda") if case["starts"] else None,
             table=_table(case["max_len"], D) if case["rope"] else None,
             out=torch.empty((case["seqs"], h, D), dtype=dt, device="cuda"), lse=torch.empty((case["seqs"], h), device="cuda"),
             ws=torch.empty(128 << 20, dtype=torch.uint8, device="cuda"))
    if kind == "step":     # the key and value of the new token, whose place in the cache holds nothing yet
        s.update(k=_keys((case["seqs"], kv, D), dt, g), v=_normal((case["seqs"], kv, D), dt, g), positions=s["lengths"] - 1)
    return s


def _filled_cache(case, pages, lengths, table, g):
    """Whole pages of keys and values, NaN after each sequence's last position."""
    buffers = _empty_cache(case, pages)
    kv, page, D = case["kv"], case["page"], case["D"]
    k, v = _keys((pages, kv, page, D), torch.bfloat16, g), _normal((pages, kv, page, D), torch.bfloat16, g)
    if case["cache"] == "bf16":
        buffers.update(k=k, v=v)
    else:
        buffers["k"], buffers["k_scales"] = _quantize(k.float(), buffers["k_scale"], "rtn")
        buffers["v"], scales = _quantize(v.float(), buffers["v_scale"], "rtn")
        buffers["v_scales"] = scales.transpose(2, 3).contiguous()
    last = torch.tensor([(i, n // page, n % page) for i, n in enumerate(lengths) if n % page], dtype=torch.int64).reshape(-1, 3).cuda()
    tail = torch.arange(page, device="cuda")[None, :] >= last[:, 2:3]
    at, slot = table[last[:, 0], last[:, 1]].long()[:, None].expand_as(tail)[tail], torch.arange(page, device="cuda").expand_as(tail)[tail]
    if case["cache"] == "bf16":
        buffers["k"][at, :, slot] = float("nan")
        buffers["v"][at, :, slot] = float("nan")
    else:
        buffers["k_scales"][at, :, slot] = 0x7F
        buffers["v_scales"][at, :, :, slot] = 0x7F
    return buffers


# ------------------------------------------------------------------------------------------------- the plain forms
def _rotate(x, positions, table, layout, inverse=False):
    """The first 2 * table.shape[2] elements of each head of x (f32), in pairs, by the angles of its position."""
    pairs = table.shape[2]
    cos, sin = table[positions.long(), 0][:, None, :], table[positions.long(), 1][:, None, :]
    if inverse:
        sin = -sin
    if layout == "half":
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
    else:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat((c, d), dim=-1) if layout == "half" else torch.stack((c, d), dim=-1).flatten(-2)
    return torch.cat((turned, x[..., 2 * pairs:]), dim=-1)


def _candidate(y, r):
    """Scale bytes, codes' values and their errors of groups y [..., 16] (f32) whose scale is r rounded to E4M3."""
    x8 = r[0].clamp(max=448.0).to(torch.float8_e4m3fn)
    p = x8.float() * r[1]
    live = x8.float() > 0
    q = y * (1.0 / torch.where(live, p, 1.0))[..., None]
    a = q.abs()
    m = torch.where(a < 2.0, torch.round(a * 2.0) * 0.5, torch.where(a < 4.0, torch.round(a), torch.round(a * 0.5) * 2.0)).clamp(max=6.0)
    c = torch.where(live[..., None], torch.copysign(m, q), 0.0)
    return x8.view(torch.uint8), c, p


def _squared_error(y, c, p):
    """Sum of (y - c p)^2 in index order, every step one fused multiply-add (one rounding of the exact binary64 value)."""
    d = torch.addcmul(y.double(), c.double(), p.double()[..., None], value=-1.0).float().double()
    e = torch.zeros_like(p)
    for i in range(16):
        e = torch.addcmul(e.double(), d[..., i], d[..., i]).float()
    return e


def _quantize(x, tensor_scale, mode):
    """NVFP4 of x [..., D] (f32) under a given tensor scale: codes [..., D / 2] and scale bytes [..., D / 16]."""
    y = x.reshape(*x.shape[:-1], -1, 16)
    top = y.abs().amax(-1)
    scales, c, p = _candidate(y, (top / (tensor_scale * 6.0), tensor_scale))
    if mode == "rtn_46":      # the group's maximum mapped to 4 where that has the smaller error
        scales4, c4, p4 = _candidate(y, (top / (tensor_scale * 4.0), tensor_scale))
        use4 = _squared_error(y, c4, p4) < _squared_error(y, c, p)
        scales, c = torch.where(use4, scales4, scales), torch.where(use4[..., None], c4, c)
    m = c.abs()
    code = torch.where(m < 2.0, m * 2.0, torch.where(m < 4.0, m + 2.0, m * 0.5 + 4.0)).to(torch.uint8) | (torch.signbit(c).to(torch.uint8) << 3)
    code = code.reshape(*x.shape[:-1], -1, 2)
    return code[..., 0] | (code[..., 1] << 4), scales


def _values(codes, scales, tensor_scale):
    """f32 values of NVFP4 codes [..., D / 2] and scale bytes [..., D / 16]."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    c = grid[torch.stack((codes & 15, codes >> 4), dim=-1).long()].reshape(*scales.shape, 16)
    return (c * scales.view(torch.float8_e4m3fn).float()[..., None] * tensor_scale).flatten(-2)


def _place(seqs, positions, page_table, page):
    positions = positions.long()
    return page_table[seqs.long(), positions // page].long(), positions % page


def _write(b, k, v, seqs, positions, page_table, mode):
    at, slot = _place(seqs, positions, page_table, b["k"].shape[2])
    if b["k_scales"] is None:
        b["k"][at, :, slot], b["v"][at, :, slot] = k.to(torch.bfloat16), v.to(torch.bfloat16)
        return
    b["k"][at, :, slot], b["k_scales"][at, :, slot] = _quantize(k, b["k_scale"], mode)
    b["v"][at, :, slot], b["v_scales"][at, :, :, slot] = _quantize(v, b["v_scale"], mode)


def _read(b, seqs, positions, page_table):
    at, slot = _place(seqs, positions, page_table, b["k"].shape[2])
    if b["k_scales"] is None:
        return b["k"][at, :, slot].float(), b["v"][at, :, slot].float()
    return (_values(b["k"][at, :, slot], b["k_scales"][at, :, slot], b["k_scale"]),
            _values(b["v"][at, :, slot], b["v_scales"][at, :, :, slot], b["v_scale"]))


def _dense(b, page_table, which):
    """f32 [seqs, kv_heads, longest, D] of all mapped pages (an unmapped one reads page 0; its positions are masked)."""
    t = b[which][page_table.clamp(min=0).long()]
    if b["k_scales"] is not None:
        scales = b[which + "_scales"][page_table.clamp(min=0).long()]
        t = _values(t, scales if which == "k" else scales.transpose(3, 4), b[which + "_scale"])
    return t.float().transpose(1, 2).flatten(2, 3)


def _attend(s):
    b, (n, h, D), kv = s["cache_buffers"], s["q"].shape, s["kv"]
    q = s["q"].float()
    if s["table"] is not None:
        q = _rotate(q, (s["lengths"] - 1).clamp(min=0), s["table"], s["layout"])
    k = _dense(b, s["page_table"], "k")
    j = torch.arange(k.shape[2], device="cuda")[None, :]
    first = torch.zeros_like(s["lengths"]) if s["starts"] is None else s["starts"]
    if s["window"]:
        first = torch.maximum(first, s["lengths"] - s["window"])
    counts = ((j >= first[:, None]) & (j < s["lengths"][:, None]))[:, None, None, :]
    scores = torch.matmul(q.view(n, kv, h // kv, D), k.transpose(2, 3).contiguous()) * s["scale"]
    del k
    scores = torch.where(counts, scores, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top) & (top < 0), 0.0, top))
    total = p.sum(-1, keepdim=True)
    v = torch.where(counts.transpose(2, 3), _dense(b, s["page_table"], "v"), 0.0)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out.view(n, h, D).to(s["q"].dtype), (top + torch.log(total)).view(n, h)


def _run_plain(s):
    kind = s["kind"]
    if kind == "rotary":
        return {"y": _rotate(s["x"].float(), s["positions"], s["table"], s["layout"], s["inverse"]).to(s["x"].dtype)}
    b = s["cache_buffers"]
    if kind in ("write", "step"):
        seqs = s["seq_ids"] if kind == "write" else torch.arange(s["seqs"], device="cuda")
        k = s["k"].float()
        if s["table"] is not None:
            k = _rotate(k, s["positions"], s["table"], s["layout"])
        _write(b, k, s["v"].float(), seqs, s["positions"], s["page_table"], s["mode"])
    if kind in ("write", "read"):
        k, v = _read(b, s["seq_ids"], s["positions"], s["page_table"])
        return {"k": k.to(s["k_out"].dtype), "v": v.to(s["v_out"].dtype)}
    out, lse = _attend(s)
    return {"out": out, "lse": lse} if kind == "attend" else {"out": out, "lse": lse, "cache": _state(b)}


def _state(b):
    return [t for t in (b["k"], b["v"], b["k_scales"], b["v_scales"]) if t is not None]


# ------------------------------------------------------------------------------------------------- one pass
def _run_own(s):
    from paper_2601_22813_amd import binding as qii
    kind = s["kind"]
    layout = qii.ROTARY_HALF if s.get("layout") == "half" else qii.ROTARY_INTERLEAVED
    if kind == "rotary":
        qii.qii_rotary(s["x"], s["positions"], s["table"], layout, s["y"], inverse=s["inverse"])
        return {"y": s["y"]}
    b = s["cache_buffers"]
    cache = qii.KVCache(b["k"], b["v"], b["k_scales"], b["v_scales"], b["k_scale"], b["v_scale"])
    if kind in ("write", "step"):
        qii.qii_kv_append(s["k"], s["v"], s["positions"], cache, s["page_table"], seqs=s.get("seq_ids"), table=s["table"], layout=layout,
                          mode=qii.RTN_46 if s["mode"] == "rtn_46" else qii.RTN)
    if kind in ("write", "read"):
        qii.qii_kv_read(cache, s["page_table"], s["positions"], s["k_out"], s["v_out"], seqs=s["seq_ids"])
        return {"k": s["k_out"], "v": s["v_out"]}
    qii.qii_paged_attention(s["q"], cache, s["page_table"], s["lengths"], s["max_len"], s["scale"], s["out"], s["ws"], lse=s["lse"],
                            starts=s["starts"], window=s["window"], table=s["table"], layout=layout)
    return {"out": s["out"], "lse": s["lse"]} if kind == "attend" else {"out": s["out"], "lse": s["lse"], "cache": _state(b)}


def run(s):
    return _run_own(s) if own else _run_plain(s)


def work(case):
    size = {"f32": 4, "bf16": 2}
    kind, D = case["kind"], case["D"]
    if kind == "rotary":
        n, per = case["tokens"], -(-case["tokens"] // case["seqs"])
        elements = n * case["heads"]
        return {"bytes": 2.0 * elements * D * size[case["dt"]] + 4 * n + 4 * case["rot"] * per, "flops": 3.0 * elements * case["rot"]}
    cached = 2 * case["kv"] * D * _element_bytes(case)       # of a position, keys and values
    if kind in ("write", "read"):
        n = sum(_lengths(dict(case, min_len=1, max_len=case["new"])))
        dense = 2 * case["kv"] * D
        if kind == "read":
            return {"bytes": n * (cached + dense * size[case["out"]] + 8), "flops": 2.0 * n * dense}
        turned = 4 * case["rot"] * min(n, case["past"] + case["new"])
        return {"bytes": n * (2 * cached + dense * (size[case["dt"]] + size[case["out"]]) + 8) + turned, "flops": 8.0 * n * dense}
    lengths = _lengths(case)
    starts = _starts(case, lengths) if case["starts"] else [0] * len(lengths)
    keys = sum(max(0, n - max(first, n - case["window"] if case["window"] else 0)) for n, first in zip(lengths, starts))
    rows = case["seqs"] * case["heads"]
    moved = keys * cached + 2 * rows * D * size[case["dt"]] + 4 * rows + 4 * keys / case["page"] + (4 * D * case["seqs"] if case["rope"] else 0)
    if kind == "step":
        moved += case["seqs"] * (2 * case["kv"] * D * size[case["dt"]] + cached)
    return {"bytes": moved, "flops": 4.0 * keys * case["heads"] * D}


# ------------------------------------------------------------------------------------------------- the same in 64 bits
def _exact_rotation(x, positions, table, layout, inverse):
    """Multiplication of a head's pairs, as complex numbers, by the table's complex numbers."""
    x, n = x.double().clone(), 2 * table.shape[2]
    t = table.double()[positions.long()]
    turn = torch.complex(t[:, 0], -t[:, 1] if inverse else t[:, 1])[:, None, :]
    even, odd = (slice(0, n // 2), slice(n // 2, n)) if layout == "half" else (slice(0, n, 2), slice(1, n, 2))
    z = torch.complex(x[..., even], x[..., odd]) * turn
    x[..., even], x[..., odd] = z.real, z.imag
    return x


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _nearest(x, grid):
    """The grid value nearest to x >= 0, of two equally near ones that with the even index."""
    i = torch.searchsorted(grid, x.contiguous()).clamp(1, len(grid) - 1)
    below, above = x - grid[i - 1], grid[i] - x
    return grid[torch.where((below < above) | ((below == above) & (i % 2 == 1)), i - 1, i)]


def _exact_nvfp4(x, tensor_scale, mode):
    """Values of x (f32 data held in 64 bits) rounded to NVFP4.  The format's rule takes its decisions in binary32, one rounding a written
    operation: each operation is done in 64 bits here and rounded to 32."""
    r32 = lambda t: t.float().double()  # noqa: E731
    e4m3 = torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127],
                        dtype=torch.float64, device=x.device)
    e2m1 = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    ts = tensor_scale.double()
    groups = x.unflatten(-1, (-1, 16))
    best = least = None
    for level in (6.0, 4.0) if mode == "rtn_46" else (6.0,):
        x8 = _nearest(r32(groups.abs().amax(-1) / r32(ts * level)).clamp(max=448.0), e4m3)
        p = r32(x8 * ts)
        c = _nearest(r32(groups.abs() * r32(1.0 / torch.where(x8 > 0, p, 1.0))[..., None]).clamp(max=6.0), e2m1) * torch.sign(groups)
        c = torch.where(x8[..., None] > 0, c, 0.0)
        e = torch.zeros_like(x8)
        for i in range(16):
            e = r32(e + r32(groups[..., i] - c[..., i] * p) ** 2)
        value = c * x8[..., None] * ts
        best = value if best is None else torch.where((e < least)[..., None], value, best)
        least = e if least is None else torch.minimum(least, e)
    return best.flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        return {"y": _exact_rotation(s["x"], s["positions"], s["table"], s["layout"], s["inverse"])}
    b = s["cache_buffers"]
    if kind == "write":
        k, v = s["k"].double(), s["v"].double()
        if s["table"] is not None:
            # the rule rounds to the cache's type from binary32: the products and their sum, each rounded to 32 bits
            n, t = 2 * s["table"].shape[2], s["table"].double()[s["positions"].long()][:, :, None, :]
            even, odd = (slice(0, n // 2), slice(n // 2, n)) if s["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
            x, y = k[..., even].clone(), k[..., odd].clone()
            k[..., even] = ((x * t[:, 0]).float().double() - (y * t[:, 1]).float().double()).float().double()
            k[..., odd] = ((y * t[:, 0]).float().double() + (x * t[:, 1]).float().double()).float().double()
        if case["cache"] == "bf16":
            return {"k": k.bfloat16().double(), "v": v.bfloat16().double()}
        return {"k": _exact_nvfp4(k, b["k_scale"], case["mode"]), "v": _exact_nvfp4(v, b["v_scale"], case["mode"])}
    if kind == "read":
        at, slot = _place(s["seq_ids"], s["positions"], s["page_table"], case["page"])
        return {"k": _exact_values(b, "k", at, slot), "v": _exact_values(b, "v", at, slot)}
    if kind == "step":
        _run_plain_write(s)
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    group = case["heads"] // case["kv"]
    for i, n in enumerate(_lengths(case)):
        first = max(_starts(case, _lengths(case))[i] if case["starts"] else 0, n - case["window"] if case["window"] else 0, 0)
        if first >= n:
            out[i], lse[i] = 0.0, float("-inf")
            continue
        j = torch.arange(first, n, device="cuda")
        at, slot = _place(torch.full_like(j, i), j, s["page_table"], case["page"])
        q = s["q"][i:i + 1].double()
        if s["table"] is not None:
            q = _exact_rotation(q, torch.tensor([n - 1], device="cuda"), s["table"], "half", False)
        k, v = (_exact_values(b, w, at, slot).transpose(0, 1).contiguous() for w in "kv")
        scores = torch.bmm(q[0].view(case["kv"], group, -1), k.transpose(1, 2).contiguous()) * s["scale"]
        total = torch.logsumexp(scores, dim=-1)
        out[i] = torch.bmm(torch.exp(scores - total[..., None]), v).flatten(0, 1)
        lse[i] = total.flatten()
    return {"out": out, "lse": lse} if kind == "attend" else {"out": out, "lse": lse, "cache": [None] * len(_state(b))}


def _run_plain_write(s):
    """The new token's entries, by the cache's own rounding rule: what the step's attention is defined on."""
    t = dict(s, kind="write", seq_ids=torch.arange(s["seqs"], device="cuda"))
    k = _rotate(t["k"].float(), t["positions"], t["table"], t["layout"])
    _write(t["cache_buffers"], k, t["v"].float(), t["seq_ids"], t["positions"], t["page_table"], t["mode"])


def _exact_values(b, which, at, slot):
    """Cached values [tokens, kv_heads, D] of the given places."""
    if b["k_scales"] is None:
        return b[which][at, :, slot].double()
    codes = b[which][at, :, slot]
    scales = b["k_scales"][at, :, slot] if which == "k" else b["v_scales"][at, :, :, slot]
    nibbles = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)
    value = torch.tensor(_E2M1 + [-x for x in _E2M1], dtype=torch.float64, device="cuda")[nibbles.long()]
    exponent, mantissa = (scales >> 3).double(), (scales & 7).double()
    x8 = torch.where(exponent > 0, (8.0 + mantissa) * torch.exp2(exponent - 10.0), mantissa * 2.0 ** -9)
    return value * x8.repeat_interleave(16, dim=-1) * b[which + "_scale"].double()
