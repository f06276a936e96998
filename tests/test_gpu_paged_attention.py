"""Attention of one new token over the paged cache against the formula in 64 bits.  Tolerances: decode_ref.attend64's, plus the
probabilities' storage (at least 11 bits kept for bf16 results, half a unit 2^-12; 22 for f32) and the result's own type."""
import numpy as np
import pytest
import torch

from paper_2601_22813_amd import binding as qii

from decode_ref import Paged, attend64, heads_view

pytestmark = pytest.mark.gpu
NVFP4, BF16 = qii.KV_NVFP4, qii.KV_BF16
bf16, f32 = torch.bfloat16, torch.float32


def ints(v):
    return None if v is None else torch.tensor(list(v), dtype=torch.int32).cuda()


def check(p, q, lengths, scale, max_length=None, starts=None, window=0, table=None, layout=0, ws="full", out=None):
    n, h, D = q.shape
    longest = max(1, max(lengths)) if max_length is None else max_length
    out = torch.full((n, h, D), float("nan"), dtype=q.dtype, device="cuda") if out is None else out
    lse = torch.full((n, h), float("nan"), device="cuda")
    need = qii.qii_paged_attention_workspace_bytes(n, h, p.kv, D, longest)
    space = None if ws is None else torch.full((max(256, need if ws == "full" else ws),), 0xFF, dtype=torch.uint8, device="cuda")
    qii.qii_paged_attention(q, p.cache, p.table, ints(lengths), longest, scale, out, space, lse=lse, starts=ints(starts), window=window,
                            table=table, layout=layout)
    torch.cuda.synchronize()
    t = None if table is None else table.cpu().numpy()
    want, want_lse, tol, tol_lse, absv = attend64(p, q.float().cpu().numpy(), lengths, scale, starts, window, t, layout, longest)
    tol = tol + absv * (2.0 ** -12 if q.dtype == bf16 else 2.0 ** -22) + 1e-30
    if q.dtype == bf16:
        tol = tol * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(want)
    else:
        tol = tol + 2.0 ** -22 * np.abs(want)
    got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])
    empty = np.isneginf(want_lse)
    assert np.array_equal(empty, np.isneginf(got_lse)) and (got[empty] == 0).all()
    assert np.all(np.abs(got_lse - want_lse)[~empty] <= tol_lse[~empty])
    return out, lse


def normal(n, h, D, dt, seed=0, **view):
    return heads_view(n, h, D, dt, torch.Generator().manual_seed(seed), **view)


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]


@pytest.mark.parametrize("kind", [NVFP4, BF16])
@pytest.mark.parametrize("dt", [bf16, f32])
@pytest.mark.parametrize("D", [16, 48, 64, 80, 128, 144, 192, 256])
def test_lengths_at_the_edges_of_tiles_and_pages(kind, dt, D):
    for page, kv, group in ((16, 2, 3), (48, 1, 8)):
        p = Paged(kind, [max(1, -(-n // page)) for n in EDGES], kv, page, D, seed=D)
        p.fill(EDGES, seed=D + 1)
        check(p, normal(len(EDGES), kv * group, D, dt), EDGES, D ** -0.5)


@pytest.mark.parametrize("kind", [NVFP4, BF16])
@pytest.mark.parametrize("kv,group", [(1, 1), (3, 1), (2, 2), (1, 7), (2, 16), (1, 17), (1, 32), (1, 40), (5, 4)])
def test_heads_share_keys_and_values(kind, kv, group):
    lengths = [200, 1, 77, 513]
    p = Paged(kind, [-(-n // 32) for n in lengths], kv, 32, 128, seed=kv)
    p.fill(lengths, seed=group)
    check(p, normal(4, kv * group, 128, bf16, seed=group), lengths, 128 ** -0.5)


@pytest.mark.parametrize("kind", [NVFP4, BF16])
@pytest.mark.parametrize("dt", [bf16, f32])
def test_long_sequences_are_split_and_joined(kind, dt):
    for lengths, kv, group, D, page in (([9001, 0, 4097, 12], 1, 4, 128, 64), ([20003], 2, 2, 64, 16), ([7000, 6999], 1, 1, 256, 128)):
        p = Paged(kind, [max(1, -(-n // page)) for n in lengths], kv, page, D, seed=7)
        p.fill(lengths, seed=8)
        q = normal(len(lengths), kv * group, D, dt, seed=9)
        a = check(p, q, lengths, D ** -0.5)
        b = check(p, q, lengths, D ** -0.5)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])          # the same bits again
        need = qii.qii_paged_attention_workspace_bytes(len(lengths), kv * group, kv, D, max(lengths))
        for ws in (None, 256, need // 3 // 256 * 256):
            check(p, q, lengths, D ** -0.5, ws=ws)
        check(p, q, lengths, D ** -0.5, max_length=p.table_np.shape[1] * page + 5000)


@pytest.mark.parametrize("lengths,group,D", [([70001], 3, 256), ([70001], 2, 80), ([66000], 5, 16), ([9000, 40000, 3], 1, 128), ([20000], 18, 64)])
def test_more_chunks_than_a_wave_joins_at_once(lengths, group, D):
    page = 256
    p = Paged(NVFP4, [max(1, -(-n // page)) for n in lengths], 1, page, D, seed=3)
    p.fill(lengths, seed=4)
    q = normal(len(lengths), group, D, f32, seed=5)
    check(p, q, lengths, D ** -0.5)
    check(p, q, lengths, D ** -0.5, window=33333, starts=[5] * len(lengths))


@pytest.mark.parametrize("kind,D", [(BF16, 64), (BF16, 128), (NVFP4, 128), (NVFP4, 256), (BF16, 256)])
@pytest.mark.parametrize("dt", [bf16, f32])
def test_a_cache_larger_than_the_gpu_keeps(kind, D, dt):
    """Buffers of more than 2^27 bytes, most of whose pages belong to nobody."""
    lengths, kv, group, page = [3000, 0, 700, 1, 257, 33], 3, 4, 32
    page_bytes = 2 * kv * page * (D * 2 if kind == BF16 else D // 16 * 9)
    p = Paged(kind, [max(1, -(-n // page)) for n in lengths], kv, page, D, seed=1, spare=(1 << 27) // page_bytes + 1)
    p.fill(lengths, seed=2)
    q = normal(len(lengths), kv * group, D, dt, seed=3)
    a = check(p, q, lengths, D ** -0.5)
    b = check(p, q, lengths, D ** -0.5, max_length=5000)
    check(p, q, lengths, D ** -0.5, window=300, starts=[100, 0, 699, 5, 2 ** 31 - 1, 0])
    assert bool((a[0][1] == 0).all()) and bool((b[0][1] == 0).all())


@pytest.mark.parametrize("kind", [NVFP4, BF16])
def test_windows_starts_and_unmapped_pages(kind):
    lengths, page, kv, D = [500, 500, 500, 100, 90, 64, 33, 1000], 16, 2, 80
    p = Paged(kind, [-(-n // page) for n in lengths], kv, page, D, seed=3)
    p.table_np[1, 4:9] = -1
    p.table_np[2, :] = -1                                                   # nothing is left of this one
    p.table_np[5, 1] = p.pages + 7
    p.table_np[7, ::2] = -1
    p.table = torch.from_numpy(p.table_np).cuda()
    p.table_np[5, 1] = -1
    p.fill(lengths, seed=4)
    q = normal(len(lengths), 6, D, bf16, seed=5)
    for starts, window in ((None, 0), (None, 1), (None, 37), (None, 10 ** 6), ([0, 60, 3, 99, 100, 64, -5, 17], 0),
                           ([450, 480, 3, 10, 5, 70, 2 ** 31 - 1, 990], 100)):
        check(p, q, lengths, 0.2, starts=starts, window=window)
    # pages before the window may be gone
    p.table_np[0, :28] = -1
    p.table = torch.from_numpy(p.table_np).cuda()
    check(p, q, lengths, 0.2, window=50)


def test_negative_and_too_long_lengths():
    p = Paged(NVFP4, [4, 4, 4, 4], 1, 16, 64, seed=0)
    p.fill([64] * 4, seed=1)
    q = normal(4, 2, 64, bf16)
    check(p, q, [-1, -2 ** 31, 64, 40], 0.125, max_length=50)               # 64 counts as 50
    check(p, q, [2 ** 31 - 1, 65, 64, 63], 0.125, max_length=2 ** 31 - 1)   # the page table ends at 64
    check(p, q, [3, 4, 5, 6], 0.125, max_length=0)


@pytest.mark.parametrize("kind", [NVFP4, BF16])
@pytest.mark.parametrize("dt", [bf16, f32])
@pytest.mark.parametrize("rot,layout", [(128, 0), (128, 1), (40, 0), (6, 1)])
def test_rotation_of_the_query(kind, dt, rot, layout):
    lengths = [1, 100, 0, 333]
    p = Paged(kind, [max(1, -(-n // 16)) for n in lengths], 2, 16, 128, seed=1)
    p.fill(lengths, seed=2)
    table = torch.empty((333, 2, rot // 2), device="cuda")
    qii.qii_rotary_table(table)
    q = normal(4, 10, 128, dt, seed=3)
    check(p, q, lengths, 0.1, table=table, layout=layout)
    short = torch.empty((100, 2, rot // 2), device="cuda")                  # the last one's position has no angle
    qii.qii_rotary_table(short)
    out = torch.zeros((4, 10, 128), dtype=dt, device="cuda")
    qii.qii_paged_attention(q, p.cache, p.table, ints(lengths), 333, 0.1, out, None, table=short, layout=layout)
    assert bool(out[3].isnan().all()) and bool(out[:3].isfinite().all())


@pytest.mark.parametrize("kind", [NVFP4, BF16])
@pytest.mark.parametrize("view", [dict(offset=1, pad=3), dict(head_stride=136), dict(heads_first=True), dict(pad=64)], ids=str)
@pytest.mark.parametrize("dt", [bf16, f32])
def test_strides(kind, view, dt):
    lengths = [70, 200]
    p = Paged(kind, [13, 13], 2, 16, 128, seed=1)
    p.fill(lengths, seed=2)
    out = normal(2, 6, 128, dt, seed=1, **view)
    check(p, normal(2, 6, 128, dt, seed=3, **view), lengths, 0.1, out=out)


def test_page_table_with_gaps_between_its_rows():
    lengths = [100, 64, 17]
    p = Paged(NVFP4, [7, 7, 7], 2, 16, 64, seed=1)
    p.fill(lengths, seed=2)
    wide = torch.full((3, 50), 10 ** 9, dtype=torch.int32, device="cuda")
    wide[:, 3:10] = p.table
    p.table = wide[:, 3:10]
    check(p, normal(3, 4, 64, bf16), lengths, 0.1)


@pytest.mark.parametrize("kind", [NVFP4, BF16])
@pytest.mark.parametrize("scale,std", [(1e-6, 1.0), (3.0, 1.0), (0.1, 100.0)])
def test_flat_and_peaked_scores(kind, scale, std):
    lengths = [700, 40]
    p = Paged(kind, [44, 44], 1, 16, 128, k_scale=0.01 * std, seed=1)
    p.fill(lengths, seed=2, std=std)
    for dt in (bf16, f32):
        check(p, normal(2, 4, 128, dt), lengths, scale)
        check(p, normal(2, 4, 128, dt) * 2.0 ** -60, lengths, scale)        # queries far below and above one
        check(p, normal(2, 4, 128, dt) * 2.0 ** 40, lengths, scale * 2.0 ** -40)


def test_what_is_not_finite_reaches_its_own_results_alone():
    lengths = [100, 100, 100, 100]
    for dt in (f32, bf16):
        p = Paged(BF16, [7] * 4, 2, 16, 64, seed=1)
        p.fill(lengths, seed=2)
        row = lambda s, j: (int(p.table_np[s, j // 16]), j % 16)   # noqa: E731
        a, b = row(0, 50)
        p.cache.k[a, 0, b, 3] = float("nan")         # a key: the rows of its heads
        a, b = row(1, 99)
        p.cache.v[a, 1, b, 5] = float("inf")         # a value: its element alone
        a, b = row(2, 0)
        p.cache.k[a, 1, b, 0] = float("inf")
        q = normal(4, 4, 64, dt, seed=5)
        q[3, 1, 7] = float("nan")                    # a query: its own row
        out = torch.empty_like(q)
        lse = torch.empty((4, 4), device="cuda")
        qii.qii_paged_attention(q, p.cache, p.table, ints(lengths), 100, 0.125, out, None, lse=lse)
        assert bool(out[0, :2].isnan().all()) and bool(lse[0, :2].isnan().all()) and bool(out[0, 2:].isfinite().all())
        assert not bool(out[1, 2:, 5].isfinite().any()) and int(out[1].isfinite().sum()) == 4 * 64 - 2 and bool(lse[1].isfinite().all())
        assert bool(out[2, :2].isfinite().all())
        assert bool(out[3, 1].isnan().all()) and bool(out[3, [0, 2, 3]].isfinite().all())


def test_scores_of_minus_infinity_alone_are_an_empty_row():
    p = Paged(BF16, [2], 1, 16, 16, seed=1)
    p.fill([20], seed=2)
    p.cache.k[torch.from_numpy(p.table_np[0]).long().cuda()] = -3e38    # sixteen of them overflow to -inf
    for dt in (f32, bf16):
        q = torch.ones((1, 2, 16), device="cuda", dtype=dt)
        out, lse = torch.empty_like(q), torch.empty((1, 2), device="cuda")
        qii.qii_paged_attention(q, p.cache, p.table, ints([20]), 20, 1.0, out, None, lse=lse)
        assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


def test_on_a_stream_of_its_own_and_replayed_from_a_graph():
    lengths, kv, D = [3000, 100, 1], 2, 128
    p = Paged(NVFP4, [200, 200, 200], kv, 16, D, seed=1)
    p.fill([3200, 3200, 3200], seed=2)
    q = normal(3, 8, D, bf16, seed=3)
    table = torch.empty((3200, 2, D // 2), device="cuda")
    qii.qii_rotary_table(table)
    length = ints(lengths)
    k, v = normal(3, kv, D, bf16, seed=4), normal(3, kv, D, bf16, seed=5)
    need = qii.qii_paged_attention_workspace_bytes(3, 8, kv, D, 3200)
    ws, out, lse = torch.empty(max(256, need), dtype=torch.uint8, device="cuda"), torch.empty_like(q), torch.empty((3, 8), device="cuda")
    pos = length - 1

    def step():
        qii.qii_kv_append(k, v, pos, p.cache, p.table, table=table)
        qii.qii_paged_attention(q, p.cache, p.table, length, 3200, 0.1, out, ws, lse=lse, table=table)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for turn in range(4):
        lens = torch.tensor([3000 + turn, 100 - turn, 1 + 700 * turn], dtype=torch.int32)
        length.copy_(lens), pos.copy_(lens - 1)
        q.copy_(normal(3, 8, D, bf16, seed=10 + turn)), k.copy_(normal(3, kv, D, bf16, seed=20 + turn))
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone(), lse.clone()
        ws.random_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(replayed[0], out) and torch.equal(replayed[1], lse)
        want, *_ = attend64(p, q.float().cpu().numpy(), lens.tolist(), 0.1, table=table.cpu().numpy())
        assert np.abs(out.float().cpu().numpy() - want).max() < 0.02 * np.abs(want).max()


def test_refusals():
    p = Paged(NVFP4, [2, 2], 2, 16, 32)
    q = torch.zeros((2, 4, 32), device="cuda")
    out = torch.full((2, 4, 32), 3.0, device="cuda")
    base = dict(q=q, cache=p.cache, page_table=p.table, lengths=ints([1, 2]), max_length=32, scale=1.0, out=out, ws=None)
    t = torch.zeros((4, 2, 17), device="cuda")
    ws = torch.empty(1024, dtype=torch.uint8, device="cuda")
    for change in (dict(q=q[:, :3], out=out[:, :3]), dict(out=out.bfloat16()), dict(q=q[..., :16], out=out[..., :16]), dict(lengths=ints([1])),
                   dict(lengths=ints([1, 2]).long()), dict(max_length=-1), dict(window=-1), dict(page_table=p.table[:1]), dict(table=t),
                   dict(starts=ints([0])), dict(lse=torch.empty((4, 2), device="cuda")), dict(ws=ws[16:]), dict(q=q.half(), out=out.half()),
                   dict(cache=qii.KVCache(p.cache.k, p.cache.v, p.cache.k_scales, p.cache.k_scales, p.cache.k_scale, p.cache.v_scale)),
                   dict(cache=qii.KVCache(p.cache.k, p.cache.v, p.cache.k_scales, p.cache.v_scales, None, p.cache.v_scale))):
        with pytest.raises((qii.QiiError, TypeError)):
            qii.qii_paged_attention(**dict(base, **change))
    assert bool((out == 3.0).all())
    qii.qii_paged_attention(q[:0], p.cache, p.table[:0], ints([]), 32, 1.0, out[:0], None)
