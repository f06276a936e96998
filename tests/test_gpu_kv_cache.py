"""The paged key-value cache: entries bit for bit against the oracle's forward-pass quantizer (NVFP4) and the nearest bf16, places left
out untouched, values read back exactly."""
import numpy as np
import pytest
import torch

from paper_2601_22813_amd import binding as qii

from decode_ref import E2M1, E4M3, Paged, heads_view, rotate

pytestmark = pytest.mark.gpu
HALF, INTER = qii.ROTARY_HALF, qii.ROTARY_INTERLEAVED
NVFP4, BF16 = qii.KV_NVFP4, qii.KV_BF16


def make_table(positions, rot):
    t = torch.empty((positions, 2, rot // 2), dtype=torch.float32, device="cuda")
    qii.qii_rotary_table(t)
    return t


def scale_of(amax, mode):
    """The tensor scale that the oracle takes for a maximum, in binary32."""
    return np.float32(amax) / np.float32(6 * (448 if mode == qii.RTN else 256))


CASES = [  # kind, counts of new tokens, pasts, kv, D, page, dt, mode, rotated elements (0: none), layout, view
    (NVFP4, [1], [0], 1, 16, 16, torch.float32, qii.RTN, 0, HALF, {}),
    (NVFP4, [1, 1, 1], [0, 15, 16], 8, 128, 16, torch.bfloat16, qii.RTN, 128, HALF, {}),
    (NVFP4, [50, 3, 64], [0, 77, 5], 2, 128, 16, torch.bfloat16, qii.RTN_46, 128, INTER, dict(pad=64)),
    (NVFP4, [33, 20], [1, 40], 3, 80, 48, torch.float32, qii.RTN, 40, INTER, {}),
    (NVFP4, [33, 20], [1, 40], 3, 80, 48, torch.float32, qii.RTN_46, 36, HALF, dict(offset=1)),
    (NVFP4, [70], [10], 5, 64, 32, torch.bfloat16, qii.RTN, 64, HALF, dict(heads_first=True)),
    (NVFP4, [19, 40], [3, 0], 1, 256, 64, torch.bfloat16, qii.RTN_46, 64, HALF, dict(head_stride=264)),
    (NVFP4, [21], [2], 4, 96, 16, torch.bfloat16, qii.RTN, 0, HALF, dict(offset=1, pad=3)),
    (NVFP4, [130], [0], 2, 112, 112, torch.float32, qii.RTN, 112, HALF, {}),
    (NVFP4, [40, 7], [0, 9], 3, 96, 32, torch.bfloat16, qii.RTN, 48, HALF, {}),        # halves that begin inside a group of 16
    (NVFP4, [40, 7], [0, 9], 3, 96, 32, torch.float32, qii.RTN_46, 80, HALF, {}),
    (NVFP4, [40], [3], 2, 96, 32, torch.bfloat16, qii.RTN, 50, INTER, {}),
    (NVFP4, [700, 433], [0, 9], 13, 128, 64, torch.bfloat16, qii.RTN, 128, HALF, dict(pad=128)),   # several heads a thread
    (BF16, [1, 1], [0, 31], 4, 128, 16, torch.bfloat16, qii.RTN, 128, HALF, {}),
    (BF16, [900, 433], [0, 9], 9, 96, 64, torch.float32, qii.RTN, 48, HALF, dict(pad=96)),
    (BF16, [37, 50], [3, 0], 2, 80, 48, torch.float32, qii.SR, 80, INTER, {}),
    (BF16, [37], [3], 1, 16, 16, torch.bfloat16, qii.RTN, 2, HALF, dict(offset=1)),
    (BF16, [64], [0], 3, 192, 64, torch.float32, qii.RTN, 0, HALF, dict(pad=7)),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_append_and_read_back(case, oracle):
    kind, news, pasts, kv, D, page, dt, mode, rot, layout, view = case
    g = torch.Generator().manual_seed(D + page)
    n = sum(news)
    k, v = heads_view(n, kv, D, dt, g, **view), heads_view(n, kv, D, dt, g, **view)
    k[:, :, 5::16] *= 6.0
    k[n // 2, 0, :16] = 0.0                                     # a group of zeros
    amax_k, amax_v = 5.0, 30.0                                  # keys saturate, values' scales fall among the small ones
    ks, vs = scale_of(amax_k, mode), scale_of(amax_v, mode)
    p = Paged(kind, [-(-(a + b) // page) for a, b in zip(pasts, news)], kv, page, D, float(ks), float(vs), seed=1)
    blank = p.snapshot()
    seqs = torch.cat([torch.full((c,), i, dtype=torch.int32) for i, c in enumerate(news)])
    pos = torch.cat([torch.arange(a, a + c, dtype=torch.int32) for a, c in zip(pasts, news)])
    order = torch.randperm(n, generator=g)                      # tokens come in any order
    seqs, pos = seqs[order], pos[order]
    table = make_table(1400, rot) if rot else None
    qii.qii_kv_append(k, v, pos.cuda(), p.cache, p.table, seqs=seqs.cuda(), table=table, layout=layout, mode=mode)
    kn, vn = (t.float().cpu().numpy() for t in (k, v))
    if rot:
        kn = rotate(kn, pos.numpy(), table.cpu().numpy(), layout, single=True)
    at = p.table_np[seqs.numpy(), pos.numpy() // page].astype(np.int64)
    slot = (pos.numpy() % page).astype(np.int64)
    ai, si = torch.from_numpy(at).cuda(), torch.from_numpy(slot).cuda()
    if kind == BF16:
        expect = [torch.from_numpy(x).bfloat16() for x in (kn, vn)]
        got = [p.cache.k[ai, :, si].cpu(), p.cache.v[ai, :, si].cpu()]
        assert torch.equal(got[0], expect[0]) and torch.equal(got[1], expect[1])
        values = [e.float().numpy() for e in expect]
    else:
        values = []
        for x, amax, ts, codes, scales in ((kn, amax_k, ks, p.cache.k[ai, :, si], p.cache.k_scales[ai, :, si]),
                                           (vn, amax_v, vs, p.cache.v[ai, :, si], p.cache.v_scales[ai, :, :, si])):
            q = oracle.quantize(np.ascontiguousarray(x.reshape(n * kv, D).astype(np.float32)), mode, rht_group=0, amax=amax)
            assert q.tensor_scale[0] == ts
            assert np.array_equal(scales.cpu().numpy().reshape(n * kv, -1), q.scales)
            assert np.array_equal(codes.cpu().numpy().reshape(n * kv, -1), q.codes)
            nib = np.stack((q.codes & 15, q.codes >> 4), -1).reshape(n, kv, D)
            values.append(((E2M1[nib] * np.repeat(E4M3[q.scales], 16, -1).reshape(n, kv, D)).astype(np.float32) * ts).astype(np.float32))
    # nothing beside the tokens' places was written
    now = p.snapshot()
    for was, t in zip(blank, now):
        if t.shape[2] == page and t.dim() == 4 and t is not (now[3] if len(now) == 4 else None):
            t[ai, :, si] = was[ai, :, si]
        else:
            t[ai, :, :, si] = was[ai, :, :, si]
        assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))
    for out in (torch.float32, torch.bfloat16):
        ko, vo = heads_view(n, kv, D, out, g, **view), torch.empty((n, kv, D), dtype=out, device="cuda")
        qii.qii_kv_read(p.cache, p.table, pos.cuda(), ko, vo, seqs=seqs.cuda())
        assert torch.equal(ko.cpu(), torch.from_numpy(values[0]).to(out)) and torch.equal(vo.cpu(), torch.from_numpy(values[1]).to(out))
        only = torch.empty((n, kv, D), dtype=out, device="cuda")
        qii.qii_kv_read(p.cache, p.table, pos.cuda(), None, only, seqs=seqs.cuda())
        assert torch.equal(only, vo)


@pytest.mark.parametrize("kind", [NVFP4, BF16])
@pytest.mark.parametrize("rot", [0, 64])
def test_tokens_without_a_place_are_left_out_and_read_as_zeros(kind, rot):
    kv, D, page = 2, 64, 16
    p = Paged(kind, [3, 2], kv, page, D, seed=2)
    p.table_np[0, 1] = -1                                       # unmapped in the middle
    p.table_np[1, 1] = p.pages                                  # no page of the cache
    p.table = torch.from_numpy(p.table_np).cuda()
    #        seq  pos
    tokens = [(0, 0), (0, 16), (0, 47), (0, 48), (1, 15), (1, 16), (1, 32), (2, 0), (-1, 0), (0, -1), (1, -2 ** 31), (0, 2 ** 31 - 1),
              (2 ** 31 - 1, 3), (0, 40)]
    written = {0, 4} if rot else {0, 2, 4, 13}                  # with the rotation's table of 40 positions 40 and 47 have no angle
    seqs, pos = (torch.tensor([t[i] for t in tokens], dtype=torch.int32).cuda() for i in (0, 1))
    n = len(tokens)
    k, v = torch.randn((n, kv, D)).cuda(), torch.randn((n, kv, D)).cuda()
    before = p.snapshot()
    qii.qii_kv_append(k, v, pos, p.cache, p.table, seqs=seqs, table=make_table(40, rot) if rot else None)
    changed = torch.zeros(p.pages, page, dtype=torch.bool)
    for a, b in zip(before[:2], p.snapshot()[:2]):
        changed |= (a.view(torch.uint8) != b.view(torch.uint8)).any(-1).any(1).cpu()
    want = torch.zeros_like(changed)
    for i in written:
        s, q = tokens[i]
        want[p.table_np[s, q // page], q % page] = True
    assert torch.equal(changed, want)
    ko, vo = torch.full((n, kv, D), 9.0).cuda(), torch.full((n, kv, D), 9.0).cuda()
    qii.qii_kv_read(p.cache, p.table, pos, ko, vo, seqs=seqs)
    gone = [i for i, (s, q) in enumerate(tokens) if not (s in (0, 1) and 0 <= q < 48 and 0 <= p.table_np[s, q // page] < p.pages)]
    assert bool((ko[gone] == 0).all()) and bool((vo[gone] == 0).all())
    assert bool((vo[sorted(written)] != 9.0).all())


@pytest.mark.parametrize("rot,layout", [(0, HALF), (32, HALF), (48, HALF), (36, HALF), (32, INTER), (6, INTER)])
def test_elements_that_do_not_turn_are_kept_as_they_are(rot, layout):
    """Zeros of either sign and infinities beside the rotated elements, whatever stands among those."""
    n, kv, D = 20, 2, 96
    p = Paged(BF16, [2], kv, 16, D)
    k = torch.randn((n, kv, D)).bfloat16().cuda()
    k[0::4, :, rot:] = -0.0
    k[1::4, :, rot:] = 0.0
    k[2::4, :, rot::3] = float("inf")
    k[2::4, :, rot + 1::3] = float("-inf")
    k[3::4, :, :rot] = float("nan")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    seqs = torch.zeros(n, dtype=torch.int32, device="cuda")
    qii.qii_kv_append(k, k, pos, p.cache, p.table, seqs=seqs, table=make_table(40, rot) if rot else None, layout=layout)
    at, slot = p.table[0, (pos // 16).long()].long(), (pos % 16).long()
    got_k, got_v = p.cache.k[at, :, slot], p.cache.v[at, :, slot]
    assert torch.equal(got_k[..., rot:].view(torch.int16), k[..., rot:].view(torch.int16))
    assert torch.equal(got_v.isnan(), k.isnan()) and torch.equal(got_v.nan_to_num(7.0), k.nan_to_num(7.0))


@pytest.mark.parametrize("kind", [NVFP4, BF16])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,D,page,n,pad", [(9, 128, 48, 3001, 0), (4, 80, 16, 5000, 80), (3, 256, 64, 1999, 5)])
def test_large_reads(kind, dt, kv, D, page, n, pad):
    """Several heads a thread, an odd number of heads, rows of another stride, places that do not exist among the others."""
    p = Paged(kind, [-(-n // page), 2], kv, page, D, seed=n)
    p.fill([n, page], seed=D)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    pos[7::13] = -1
    seqs = torch.zeros(n, dtype=torch.int32, device="cuda")
    ko, vo = (heads_view(n, kv, D, dt, torch.Generator().manual_seed(0), pad=pad) for _ in range(2))
    qii.qii_kv_read(p.cache, p.table, pos, ko, vo, seqs=seqs)
    for got, want in zip((ko, vo), p.values(0, np.arange(n))):
        want = torch.from_numpy(want).float().to(dt)            # (the product of both scales and a code, rounded to f32 and then to dt)
        want[7::13] = 0
        assert torch.equal(got.cpu(), want)


def test_positions_past_32_bits_of_bytes():
    """A cache of more than 4 GiB on each side: the last pages' addresses."""
    kv, D, page = 4, 256, 64
    pages = (1 << 32) // (kv * D * page * 2) + 40
    p = Paged(BF16, [1], kv, page, D, seed=0)
    cache = qii.KVCache.empty(BF16, pages, kv, page, D)
    table = torch.tensor([[pages - 1, 0, pages - 33]], dtype=torch.int32, device="cuda")
    n = 3 * page
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    k, v = torch.randn((n, kv, D), device="cuda").bfloat16(), torch.randn((n, kv, D), device="cuda").bfloat16()
    qii.qii_kv_append(k, v, pos, cache, table, seqs=torch.zeros(n, dtype=torch.int32, device="cuda"))
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    qii.qii_kv_read(cache, table, pos, ko, vo, seqs=torch.zeros(n, dtype=torch.int32, device="cuda"))
    assert torch.equal(ko, k) and torch.equal(vo, v)
    assert torch.equal(cache.k[pages - 1].transpose(0, 1), k[:page])
    q = torch.randn((1, 8, D), device="cuda").bfloat16()
    out = torch.empty_like(q)
    qii.qii_paged_attention(q, cache, table, torch.tensor([n - 5], dtype=torch.int32, device="cuda"), n, 0.0625, out, None)
    kk, vv = k[:n - 5].double().repeat_interleave(2, 1), v[:n - 5].double().repeat_interleave(2, 1)
    w = torch.softmax((kk * q.double()).sum(-1) * 0.0625, 0)
    assert float((out.double() - (w[..., None] * vv).sum(0)).abs().max()) < 0.01
    del p


def test_refusals():
    p = Paged(NVFP4, [2], 2, 16, 32)
    x = torch.zeros((3, 2, 32), device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    seqs = torch.zeros(3, dtype=torch.int32, device="cuda")
    before = p.snapshot()
    bad = [dict(k=x[:2]), dict(v=x.bfloat16()), dict(k=x.half(), v=x.half()), dict(positions=pos.long()), dict(seqs=seqs[:2]), dict(mode=qii.SR),
           dict(mode=qii.MS_EDEN), dict(k=x[:, :1], v=x[:, :1]), dict(page_table=p.table.long()), dict(table=make_table(4, 34)),
           dict(table=make_table(4, 32), layout=5), dict(page_table=p.table[0])]
    for change in bad:
        args = dict(dict(k=x, v=x, positions=pos, cache=p.cache, page_table=p.table, seqs=seqs), **change)
        with pytest.raises((qii.QiiError, TypeError)):
            qii.qii_kv_append(**args)
    for change in (dict(k_out=None, v_out=None), dict(k_out=x[:2]), dict(v_out=x.bfloat16()), dict(positions=pos.long())):
        args = dict(dict(cache=p.cache, page_table=p.table, positions=pos, k_out=x, v_out=x.clone(), seqs=seqs), **change)
        with pytest.raises((qii.QiiError, TypeError)):
            qii.qii_kv_read(**args)
    for shape in ((2, 2, 24, 32), (2, 2, 16, 24), (2, 2, 8, 32)):
        with pytest.raises(qii.QiiError):
            cache = qii.KVCache.empty(BF16, *shape)
            y = torch.zeros((3, 2, shape[3]), device="cuda")
            qii.qii_kv_append(y, y, pos, cache, p.table, seqs=seqs)
    assert all(torch.equal(a, b) for a, b in zip(before, p.snapshot())) and bool((x == 0).all())
    qii.qii_kv_append(x[:0], x[:0], pos[:0], p.cache, p.table, seqs=seqs[:0])
    qii.qii_kv_read(p.cache, p.table, pos[:0], x[:0], x[:0], seqs=seqs[:0])
