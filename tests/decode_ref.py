"""Plain numpy definitions of the operators between a decoder's projections, in 64 bits, and inputs for their tests."""
import numpy as np
import torch

from paper_2601_22813_amd import binding as qii

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)])
E4M3[127] = np.nan
EPS = 2.0 ** -24                      # half a unit in the last place of binary32, relative


def table64(positions, rot, base=10000.0, scaling=0, factor=1.0, original=0.0, fast=32.0, slow=1.0, magnitude=1.0):
    i = np.arange(rot // 2)
    if scaling == qii.ROTARY_SCALING_BASE:
        base = base * factor ** (rot / max(rot - 2, 1))
    f = base ** (-2.0 * i / rot)
    if scaling == qii.ROTARY_SCALING_LINEAR:
        f = f / factor
    if scaling == qii.ROTARY_SCALING_BY_PARTS:
        ramp = np.clip((original * f / (2 * np.pi) - slow) / (fast - slow), 0.0, 1.0)
        f = (1 - ramp) * f / factor + ramp * f
    a = np.arange(positions)[:, None] * f
    return magnitude * np.stack((np.cos(a), np.sin(a)), axis=1)


def pairs_of(rot, layout):
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if layout == qii.ROTARY_HALF else (2 * i, 2 * i + 1)


def rotate(x, positions, table, layout, inverse=False, single=False):
    """x [tokens, heads, D] (numpy).  single: binary32, a rounding for each written operation; else the type of x and table."""
    x = np.array(x, dtype=np.float32 if single else np.float64)
    t = np.asarray(table, dtype=x.dtype)[positions]
    c, s = t[:, None, 0], t[:, None, 1] * (-1 if inverse else 1)
    a, b = pairs_of(2 * table.shape[2], layout)
    p, q = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = p * c - q * s, q * c + p * s
    return x


def heads_view(n, h, D, dt, g, head_stride=None, pad=0, offset=0, heads_first=False):
    """A [n, h, D] view with strides of its own into a buffer of normal numbers."""
    hs = head_stride or D
    if heads_first:
        buf = torch.randn(h * n * D + offset, generator=g).to(dt).cuda()
        return buf[offset:].view(h, n, D).transpose(0, 1)
    ts = h * hs + pad
    buf = torch.randn(n * ts + offset, generator=g).to(dt).cuda()
    return torch.as_strided(buf, (n, h, D), (ts, hs, 1), offset)


class Paged:
    """A cache whose sequences have the given page counts, in pages of no order; whatever is not written holds NaN."""

    def __init__(self, kind, counts, kv, page, D, k_scale=0.01, v_scale=0.005, seed=0, spare=3):
        rng = np.random.default_rng(seed)
        total = int(sum(counts)) + spare
        width = max(1, max(counts))
        order = rng.permutation(total)[: total - spare]
        self.table_np = np.full((len(counts), width), -1, dtype=np.int32)
        at = 0
        for i, c in enumerate(counts):
            self.table_np[i, :c] = order[at:at + c]
            at += c
        self.kind, self.kv, self.page, self.D, self.pages = kind, kv, page, D, total
        f = lambda v: torch.full((1,), v, dtype=torch.float32, device="cuda")   # noqa: E731
        self.cache = qii.KVCache.empty(kind, total, kv, page, D, f(k_scale), f(v_scale))
        if kind == qii.KV_BF16:
            self.cache.k.fill_(float("nan")), self.cache.v.fill_(float("nan"))
        else:
            self.cache.k.fill_(0x77), self.cache.v.fill_(0xFF), self.cache.k_scales.fill_(0x7F), self.cache.v_scales.fill_(0xFF)
        self.table = torch.from_numpy(self.table_np).cuda()

    def snapshot(self):
        c = self.cache
        return [t.clone() for t in (c.k, c.v, c.k_scales, c.v_scales) if t is not None]

    def fill(self, lengths, seed=0, std=1.0):
        """Random entries at the first lengths[i] positions of each sequence."""
        g = torch.Generator().manual_seed(seed)
        for i, n in enumerate(lengths):
            j = np.arange(n)
            at, slot = self.table_np[i, j // self.page], j % self.page
            ok = at >= 0
            at, slot = torch.from_numpy(at[ok].astype(np.int64)).cuda(), torch.from_numpy(slot[ok]).cuda()
            m = len(at)
            for which, buf in (("k", self.cache.k), ("v", self.cache.v)):
                if self.kind == qii.KV_BF16:
                    buf[at, :, slot] = (torch.randn((m, self.kv, self.D), generator=g) * std).bfloat16().cuda()
                    continue
                buf[at, :, slot] = torch.randint(0, 256, (m, self.kv, self.D // 2), generator=g, dtype=torch.uint8).cuda()
                # scales from the smallest (subnormal, zero) to ordinary ones
                b = torch.randint(40, 80, (m, self.kv, self.D // 16), generator=g, dtype=torch.uint8)
                b[torch.rand(b.shape, generator=g) < 0.05] = 0
                b[torch.rand(b.shape, generator=g) < 0.05] = 3
                if which == "k":
                    self.cache.k_scales[at, :, slot] = b.cuda()
                else:
                    self.cache.v_scales[at, :, :, slot] = b.cuda()

    def values(self, seq, positions):
        """float64 keys and values [n, kv, D] of mapped positions."""
        at, slot = self.table_np[seq, positions // self.page], positions % self.page
        c, out = self.cache, []
        for buf, scales, ts, value in ((c.k, c.k_scales, c.k_scale, False), (c.v, c.v_scales, c.v_scale, True)):
            a, s = torch.from_numpy(at.astype(np.int64)).cuda(), torch.from_numpy(slot).cuda()
            x = buf[a, :, s].cpu()
            if self.kind == qii.KV_BF16:
                out.append(x.double().numpy())
                continue
            codes = x.numpy()
            nib = np.stack((codes & 15, codes >> 4), axis=-1).reshape(*codes.shape[:-1], -1)
            b = (scales[a, :, :, s] if value else scales[a, :, s]).cpu().numpy()
            out.append(E2M1[nib] * np.repeat(E4M3[b & 127], 16, axis=-1) * float(ts.item()))
        return out


def attend64(p, q, lengths, scale, starts=None, window=0, table=None, layout=0, max_length=1 << 30):
    """(out, lse, tol_out, tol_lse) in float64.  The tolerances are of binary32 sums of the same terms in any order, one rounding each:
      a score      (D + 16) eps * scale * sum_d |q_d k_d|           (products, their sum, q's rotation, the scale) = ds
      an exponent  the score's error, and that of an argument of |s - max| <= 100 in units of log2 (below that a term is nothing)
      out          the relative error of each weight, and (n + 32) eps for the sums, times sum_j p_j |v_j|
    plus that of the probabilities' storage and of the result's type, which the caller adds."""
    n, h, D = q.shape
    group = h // p.kv
    out, lse = np.zeros((n, h, D)), np.full((n, h), -np.inf)
    tol, tol_lse = np.zeros((n, h, D)), np.zeros((n, h))
    absv = np.zeros((n, h, D))
    for i in range(n):
        length = min(max(int(lengths[i]), 0), max_length, p.table_np.shape[1] * p.page)
        first = max(0 if starts is None else int(starts[i]), length - window if window else 0, 0)
        j = np.arange(first, max(first, length))
        j = j[(p.table_np[i, j // p.page] >= 0) & (p.table_np[i, j // p.page] < p.pages)]
        if len(j) == 0:
            continue
        qi = q[i:i + 1].astype(np.float64)
        if table is not None:
            qi = rotate(qi, np.array([length - 1]), table, layout)
        k, v = p.values(i, j)
        for head in range(h):
            kh, vh = k[:, head // group], v[:, head // group]
            s = kh @ qi[0, head] * scale
            ds = (D + 16) * EPS * scale * np.max(np.abs(kh) @ np.abs(qi[0, head]))
            top = s.max()
            w = np.exp(s - top)
            total = w.sum()
            w /= total
            rel = 2 * ds + 2 * 150 * EPS + (len(j) + 32) * EPS
            out[i, head], lse[i, head] = w @ vh, top + np.log(total)
            absv[i, head] = w @ np.abs(vh)
            tol[i, head], tol_lse[i, head] = rel * absv[i, head], rel + 4 * EPS * (abs(top) + np.log(len(j)) + 1)
    return out, lse, tol, tol_lse, absv
