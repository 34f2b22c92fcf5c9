"""The block operators from their definitions, in fp64 on the CPU (torch tensors in,
torch tensors out).  Test infrastructure: nothing here is shared with the GPU path."""

import math

import torch


def turned(x, pos, freqs, sections, heads, neighbours=False, back=False):
    """Rotary positions pair by pair.  Returns (out, |u| + |v| of each entry's pair, the
    angle's size in turns): x [n, heads, hd], pos [n, axes]."""
    out, size, turns = x.double().clone(), x.double().abs(), torch.zeros(x.shape, dtype=torch.float64)
    axes = [a for a, s in enumerate(sections) for _ in range(s)]
    pairs = len(axes)
    for f, a in enumerate(axes):
        angle = pos[:, a].double() * float(freqs[f]) * (-1 if back else 1)
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        i, j = (2 * f, 2 * f + 1) if neighbours else (f, f + pairs)
        u, v = x[:, :heads, i].double(), x[:, :heads, j].double()
        out[:, :heads, i], out[:, :heads, j] = u * c - v * s, v * c + u * s
        for k in (i, j):
            size[:, :heads, k] = u.abs() + v.abs()
            turns[:, :heads, k] = angle.abs()[:, None] / (2 * math.pi)
    return out, size, turns


def philox(counter, key):
    """Philox 4x32 in ten rounds: four words from four words and a key of two."""
    (a, b, c, d), (k, l) = counter, key
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = (q >> 32) ^ b ^ k, q & 0xFFFFFFFF, (p >> 32) ^ d ^ l, p & 0xFFFFFFFF
        k, l = (k + 0x9E3779B9) & 0xFFFFFFFF, (l + 0xBB67AE85) & 0xFFFFFFFF
    return a, b, c, d


def kept(n, d, p, seed, site=0, row0=0):
    """[n, d]: what dropout multiplies with, entry by entry."""
    cut = int(round(float(torch.tensor(p, dtype=torch.float32)) * 65536))  # (p as the interface has it; ties to even)
    m = torch.zeros((n, d), dtype=torch.float64)
    seed &= (1 << 64) - 1
    for r in range(n):
        for c in range(d // 8):
            at = (row0 + r) * (d // 8) + c
            words = philox((at & 0xFFFFFFFF, at >> 32, site, 0), (seed & 0xFFFFFFFF, seed >> 32))
            bits = sum(w << 32 * i for i, w in enumerate(words))
            for e in range(8):
                if (bits >> 16 * e & 0xFFFF) >= cut:
                    m[r, 8 * c + e] = 65536 / (65536 - cut)
    return m


def _unit(t, size, rms, eps):
    """(N(t), its factor, what an error of t's terms `size` may do to it): an error of t
    moves the entry, the mean, and by the factor all entries of the row."""
    mean = 0.0 if rms else t.mean(-1, keepdim=True)
    r = ((t - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    u = (t - mean) * r
    s = size * r if rms else (size + size.mean(-1, keepdim=True)) * r
    return u, r, s + u.abs() * (1 + s.square().mean(-1, keepdim=True).sqrt())


def add_norm(x, y=None, gate=None, post_w=None, post_b=None, pre_w=None, pre_b=None, rms=False, eps=1e-5, alpha=1.0,
             mask=None, dh=None, dz=None):
    """h, z and with dh or dz all gradients, by the formulas; for each result also
    "<name>_abs": the sum of the absolute values of what it is computed from, which fp32
    errors are relative to.  mask: what dropout multiplies with."""
    f = lambda t: None if t is None else t.double()  # noqa: E731
    x, y, gate, w1, b1, w2, b2, dh, dz = (f(t) for t in (x, y, gate, post_w, post_b, pre_w, pre_b, dh, dz))
    one = torch.ones((), dtype=torch.float64)
    w1_, w2_, gate_ = (one if t is None else t for t in (w1, w2, gate))
    m = one if mask is None else mask
    r = {}
    h, habs = x, x.abs()
    if y is not None:
        v, vabs, r1 = y, y.abs(), one
        if w1 is not None:
            v, r1, vabs = _unit(y, y.abs(), rms, eps)
        t = (v * w1_ + (0 if b1 is None else b1)) * m
        tabs = (vabs * w1_.abs() + (0 if b1 is None else b1.abs())) * m
        h, habs = alpha * x + gate_ * t, (alpha * x).abs() + gate_.abs() * tabs
        r["h"], r["h_abs"] = h, habs
    if w2 is not None:
        k, r2, kabs = _unit(h, habs, rms, eps)
        r["z"] = k * w2 + (0 if b2 is None else b2)
        r["z_abs"] = kabs * w2.abs() + (0 if b2 is None else b2.abs())
    if dh is None and dz is None:
        return r
    mean = lambda a: a.mean(-1, keepdim=True)  # noqa: E731
    e = torch.zeros_like(x) if dh is None else dh
    eabs = e.abs()
    if dz is not None:
        g = dz * w2
        e = e + r2 * (g - k * mean(g * k) - (0 if rms else mean(g)))
        ga = g.abs()
        eabs = eabs + r2 * (ga + kabs * mean(ga * kabs) + (0 if rms else mean(ga))) * (1 + mean(kabs.square()).sqrt())
        r["dpre_w"], r["dpre_w_abs"] = (dz * k).sum(0), (dz.abs() * kabs).sum(0)
        r["dpre_b"], r["dpre_b_abs"] = dz.sum(0), dz.abs().sum(0)
    r["dx"], r["dx_abs"] = alpha * e, abs(alpha) * eabs
    if y is None:
        return r
    r["dgate"], r["dgate_abs"] = (e * t).sum(0), (eabs * tabs).sum(0)
    s, sabs = e * gate_ * m, eabs * gate_.abs() * m
    if w1 is None:
        r["dy"], r["dy_abs"] = s, sabs
        return r
    r["dpost_w"], r["dpost_w_abs"] = (s * v).sum(0), (sabs * vabs).sum(0)
    r["dpost_b"], r["dpost_b_abs"] = s.sum(0), sabs.sum(0)
    q, qa = s * w1, sabs * w1.abs()
    r["dy"] = r1 * (q - v * mean(q * v) - (0 if rms else mean(q)))
    r["dy_abs"] = r1 * (qa + vabs * mean(qa * vabs) + (0 if rms else mean(qa))) * (1 + mean(vabs.square()).sqrt())
    return r


def fp8(x, block=128):
    """(values [n, k] in units of their block's power of two, exponents [n, ceil(k / 128)]
    with 127 added) of x's rows in 8-bit floats, entry by entry; 255: not finite."""
    n, k = x.shape
    y = x.double()
    q = torch.zeros((n, k), dtype=torch.float64)
    exps = torch.zeros((n, (k + block - 1) // block), dtype=torch.int64)
    for r in range(n):
        for c in range(exps.shape[1]):
            s = slice(c * block, min(k, (c + 1) * block))
            row = y[r, s]
            if not torch.isfinite(row).all():
                exps[r, c] = 255
                q[r, s] = math.nan
                continue
            top, e = float(row.abs().max()), -126
            while top / 2.0 ** e > 448:
                e += 1
            exps[r, c] = e + 127
            q[r, s] = torch.tensor([_nearest(float(t) / 2.0 ** e) for t in row], dtype=torch.float64)
    return q, exps


def _nearest(t):
    """The nearest number of three bits after the leading one, down to steps of 2^-9."""
    step = 2.0 ** (max(math.frexp(t)[1] - 1, -6) - 3)
    return math.copysign(round(abs(t) / step) * step, t)  # (Python rounds ties to even)


def unfp8(q, exps, block=128):
    e = exps.repeat_interleave(block, 1)[:, :q.shape[1]].double()
    return torch.where(e == 255, math.nan, q * torch.exp2(e - 127))
