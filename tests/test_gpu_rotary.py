"""Rotary positions against their formulas: bit for bit against binary32 with a rounding for each written operation, to a derived
bound against 64 bits, the gradient against differences."""
import numpy as np
import pytest
import torch

from paper_2601_22813_amd import binding as qii

from decode_ref import EPS, heads_view, pairs_of, rotate, table64

pytestmark = pytest.mark.gpu
HALF, INTER = qii.ROTARY_HALF, qii.ROTARY_INTERLEAVED


def to_np(t):
    return t.float().cpu().numpy()


def make_table(positions, rot, **kw):
    t = torch.empty((positions, 2, rot // 2), dtype=torch.float32, device="cuda")
    qii.qii_rotary_table(t, **kw)
    return t


@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling=qii.ROTARY_SCALING_LINEAR, factor=8.0),
                                dict(scaling=qii.ROTARY_SCALING_BASE, factor=4.0),
                                dict(scaling=qii.ROTARY_SCALING_BY_PARTS, factor=16.0, original_positions=4096.0, magnitude=1.2772588722239782),
                                dict(scaling=qii.ROTARY_SCALING_BY_PARTS, factor=4.0, original_positions=64.0, turns_fast=8.0, turns_slow=0.0)])
@pytest.mark.parametrize("positions,rot", [(1, 2), (37, 2), (1000, 48), (70001, 128), (20000, 6)])
def test_table_is_the_rounded_cosine_and_sine_of_the_scaled_angle(kw, positions, rot):
    got = to_np(make_table(positions, rot, **kw)).astype(np.float64)
    names = {"original_positions": "original", "turns_fast": "fast", "turns_slow": "slow"}
    want = table64(positions, rot, **{names.get(k, k): v for k, v in kw.items()})
    # one rounding to binary32, and the angle's error in 64 bits: a few 2^-53 of at most 70001 radians
    assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want) * 1.0001 + 8 * 70001 * 2.0 ** -52)


CASES = [  # tokens, heads, D, rot, layout, view
    (1, 1, 2, 2, HALF, {}), (1, 1, 1 + 2, 2, INTER, {}), (3, 5, 64, 64, HALF, {}), (3, 5, 64, 64, INTER, {}),
    (33, 4, 128, 128, HALF, dict(pad=256)), (33, 4, 128, 128, INTER, dict(pad=256)), (17, 3, 96, 48, INTER, dict(head_stride=104)),
    (17, 3, 96, 48, HALF, dict(head_stride=97, pad=5)), (9, 2, 80, 40, HALF, dict(offset=1)), (9, 2, 80, 36, INTER, dict(offset=3)),
    (65, 7, 50, 50, HALF, {}), (65, 7, 33, 6, INTER, {}), (40, 6, 128, 64, HALF, dict(heads_first=True)), (40, 6, 256, 32, HALF, {}),
    (300, 40, 112, 112, HALF, {}), (2, 1, 512, 512, INTER, {}), (1025, 3, 128, 16, HALF, dict(pad=8)), (7, 2, 48, 24, HALF, dict(pad=16)),
]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_bit_for_bit_and_in_place(case, dt, inverse):
    n, h, D, rot, layout, view = case
    g = torch.Generator().manual_seed(n * 1000 + D)
    x = heads_view(n, h, D, dt, g, **view)
    table = make_table(600, rot, magnitude=1.1)
    pos = torch.randint(0, 600, (n,), generator=g, dtype=torch.int32)
    y = torch.full((n, h, D), float("nan"), dtype=dt, device="cuda")
    before = x.clone()
    qii.qii_rotary(x, pos.cuda(), table, layout, y, inverse=inverse)
    t = table.cpu().numpy()
    want = torch.from_numpy(rotate(to_np(x), pos.numpy(), t, layout, inverse, single=True)).to(dt)
    assert torch.equal(y.cpu(), want) and torch.equal(x, before)
    # against 64 bits: two products and a sum, half a unit each; bf16 once more
    exact = rotate(to_np(x), pos.numpy(), t, layout, inverse)
    a, b = pairs_of(rot, layout)
    size = np.abs(to_np(x)).astype(np.float64)
    bound = size.copy()
    bound[..., a] = bound[..., b] = 1.1 * (size[..., a] + size[..., b])
    tol = 3 * EPS * bound + (2.0 ** -8 * np.abs(exact) if dt == torch.bfloat16 else 0)
    assert np.all(np.abs(to_np(y).astype(np.float64) - exact) <= tol)
    qii.qii_rotary(x, pos.cuda(), table, layout, x, inverse=inverse)      # in place, and nothing beside the view's elements
    assert torch.equal(x, y)


def test_what_lies_between_the_elements_of_the_views_is_untouched():
    g = torch.Generator().manual_seed(5)
    buf = torch.randn(50, 400, generator=g).bfloat16().cuda()
    out = torch.full((50, 500), 7.0, dtype=torch.bfloat16, device="cuda")
    x, y = buf[:, 8:8 + 3 * 96].view(50, 3, 96), out[:, 16:16 + 3 * 112].view(50, 3, 112)[..., :96]
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    qii.qii_rotary(x, pos, make_table(50, 96), HALF, y)
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[:, 16:16 + 3 * 112].view(50, 3, 112)[..., :96] = False
    assert bool((out[rest] == 7.0).all()) and not bool((y == 7.0).all(-1).any())


@pytest.mark.parametrize("D,rot,layout", [(64, 64, HALF), (64, 32, INTER), (30, 10, HALF)])
def test_padding_gives_zeros_and_positions_beyond_the_table_nan(D, rot, layout):
    x = torch.full((6, 2, D), float("inf"), device="cuda")
    x[4:] = 1.0
    pos = torch.tensor([-1, -2 ** 31, 10, 2 ** 31 - 1, 9, 0], dtype=torch.int32, device="cuda")
    for inverse in (False, True):
        y = torch.empty_like(x)
        qii.qii_rotary(x, pos, make_table(10, rot), layout, y, inverse=inverse)
        assert bool((y[:2] == 0).all()) and bool(y[2:4].isnan().all()) and bool(y[4:].isfinite().all())


@pytest.mark.parametrize("layout", [HALF, INTER])
@pytest.mark.parametrize("rot", [64, 24])
def test_gradient_against_differences(layout, rot):
    """L(x) = <w, rotary(x)> is linear: (L(x + e d) - L(x - e d)) / 2e has no error but that of binary32."""
    g = torch.Generator().manual_seed(rot)
    n, h, D = 12, 3, 64
    x, w, d = (torch.randn((n, h, D), generator=g).cuda() for _ in range(3))
    pos = torch.randint(-1, 300, (n,), generator=g, dtype=torch.int32).cuda()
    table = make_table(300, rot, magnitude=0.9)
    ys = [torch.empty_like(x) for _ in range(2)]
    e = 0.5
    for sign, y in zip((1, -1), ys):
        qii.qii_rotary(x + sign * e * d, pos, table, layout, y)
    difference = float(((ys[0].double() - ys[1].double()) * w.double()).sum()) / (2 * e)
    dx = torch.empty_like(x)
    qii.qii_rotary(w, pos, table, layout, dx, inverse=True)
    # every element of a y and of dx within 3 eps of at most 2 * 1.27 (|x| + e |d|)
    tol = 3 * EPS * float((w.abs() * (x.abs().max() + d.abs().max())).double().sum()) * 4 + 3 * EPS * 3 * float(d.abs().double().sum()) * float(w.abs().max())
    assert abs(difference - float((dx.double() * d.double()).sum())) <= tol


def test_many_heads_and_tokens_of_a_fused_projection():
    """q and k of a [tokens, 6144] projection, and more elements than a grid has threads at one each."""
    n = 2300
    qkv = torch.randn((n, 6144), device="cuda").bfloat16()
    pos = (torch.arange(n, device="cuda") % 700).to(torch.int32)
    table = make_table(700, 128)
    y = torch.empty((n, 32, 128), dtype=torch.bfloat16, device="cuda")
    x = qkv[:, :4096].view(n, 32, 128)
    qii.qii_rotary(x, pos, table, HALF, y)
    c, s = table[pos.long()][:, None, 0], table[pos.long()][:, None, 1]
    a, b = x.float()[..., :64], x.float()[..., 64:]
    assert torch.equal(y, torch.cat((a * c - b * s, b * c + a * s), -1).bfloat16())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,rot,layout", [(128, 128, HALF), (128, 64, INTER), (96, 48, HALF), (256, 128, HALF), (80, 40, INTER)])
@pytest.mark.parametrize("inverse", [False, True])
def test_large_tensors_are_turned_as_small_ones(dt, D, rot, layout, inverse):
    """The same bits from one call of more than 2^22 elements, into a view and in place, as from calls of few tokens."""
    n, h = 5 * 2 ** 22 // (4 * 9 * D), 9
    x = torch.randn((n, h, D), device="cuda").to(dt)
    pos = (torch.arange(n, device="cuda") % 701 - 1).to(torch.int32)        # (padding among them)
    table = make_table(690, rot)                                            # (and positions that it does not have)
    want = torch.empty_like(x)
    for i in range(0, n, 200):
        qii.qii_rotary(x[i:i + 200], pos[i:i + 200], table, layout, want[i:i + 200], inverse=inverse)
    bits = torch.int16 if dt == torch.bfloat16 else torch.int32
    room = torch.zeros((n, h + 2, D), device="cuda", dtype=dt)
    qii.qii_rotary(x, pos, table, layout, room[:, 1:-1], inverse=inverse)
    same = (room[:, 1:-1].view(bits) == want.view(bits)) | (room[:, 1:-1].isnan() & want.isnan())
    assert bool(same.all()) and bool((room[:, 0] == 0).all()) and bool((room[:, -1] == 0).all())
    qii.qii_rotary(x, pos, table, layout, x, inverse=inverse)
    assert bool(((x.view(bits) == want.view(bits)) | (x.isnan() & want.isnan())).all())


def test_empty_calls_and_refusals():
    x = torch.zeros((4, 2, 32), device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    t = make_table(8, 32)
    qii.qii_rotary(x[:0], pos[:0], t, HALF, x[:0])
    qii.qii_rotary(x[:, :0], pos, t, HALF, x[:, :0])
    for args in ((x, pos.long(), t, HALF, x), (x, pos, t.double(), HALF, x), (x.half(), pos, t, HALF, x.half())):
        with pytest.raises((TypeError, qii.QiiError)):
            qii.qii_rotary(*args)
    for args in ((x, pos[:3], t, HALF, x), (x, pos, t, 2, x), (x, pos, make_table(8, 34), HALF, x), (x, pos, t, HALF, x.bfloat16()),
                 (x, pos, t, HALF, x[:3]), (x.transpose(1, 2), pos, t, HALF, x), (x[0], pos, t, HALF, x[0])):
        with pytest.raises(qii.QiiError):
            qii.qii_rotary(*args)
    assert bool((x == 0).all())
