"""The text tower's operators from their definitions, in fp64 on the CPU (torch
tensors in, torch tensors out).  Test infrastructure: nothing here is shared
with the GPU path."""

import math

import torch


def attention(q, k, v, cu_q, cu_k, causal, scale, dout=None):
    """Packed attention, sequence by sequence and head by head.

    q [tq, heads, hd], k, v [tk, kv, hd], offsets as lists.  Returns a dict: out,
    lse [heads, tq], and with dout dq, dk, dv; and for error bounds of sums that
    round the weights p and ds to fewer bits
      out_abs  sum_j p |v|             dv_abs  sum_i p |do|
      dq_abs   scale sum_j |ds| |k|    dk_abs  scale sum_i |ds| |q|
    and of sums whose D_i is off by |do_i| . |o_i| (dq_dlt, dk_dlt), or whose scores
    are off by |q_i| . |k_j| scale (as relative error of p: *_s)."""
    q, k, v = q.double(), k.double(), v.double()
    tq, heads, hd = q.shape
    tk, kv, _ = k.shape
    g = heads // kv
    r = {n: torch.zeros_like(q) for n in ("out", "out_abs", "dq", "dq_abs", "dq_dlt")}
    r |= {n: torch.zeros_like(k) for n in ("dk", "dk_abs", "dk_dlt", "dv", "dv_abs")}
    r["lse"] = torch.full((heads, tq), -math.inf, dtype=torch.float64)
    do_all = None if dout is None else dout.double()
    for z in range(len(cu_q) - 1):
        a, b = slice(cu_q[z], cu_q[z + 1]), slice(cu_k[z], cu_k[z + 1])
        m, n = a.stop - a.start, b.stop - b.start
        if m == 0 or n == 0:
            continue
        seen = torch.ones((m, n), dtype=torch.bool)
        if causal:
            seen = torch.arange(n)[None, :] <= torch.arange(m)[:, None] + (n - m)
        some = seen.any(1)
        for h in range(heads):
            Q, K, V = q[a, h], k[b, h // g], v[b, h // g]
            s = torch.where(seen, scale * (Q @ K.T), -math.inf)
            lse = torch.logsumexp(s, 1)
            p = torch.where(seen & some[:, None], torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
            o = p @ V
            r["lse"][h, a] = torch.where(some, lse, -math.inf)
            r["out"][a, h] = o
            r["out_abs"][a, h] = p @ V.abs()
            if do_all is None:
                continue
            do = do_all[a, h]
            dp = do @ V.T
            ds = p * (dp - (do * o).sum(1, keepdim=True))
            dlt = p * (do.abs() * o.abs()).sum(1, keepdim=True)
            r["dq"][a, h] = scale * ds @ K
            r["dq_abs"][a, h] = scale * ds.abs() @ K.abs()
            r["dq_dlt"][a, h] = scale * dlt @ K.abs()
            r["dk"][b, h // g] += scale * ds.T @ Q
            r["dk_abs"][b, h // g] += scale * ds.abs().T @ Q.abs()
            r["dk_dlt"][b, h // g] += scale * dlt.T @ Q.abs()
            r["dv"][b, h // g] += p.T @ do
            r["dv_abs"][b, h // g] += p.T @ do.abs()
    return r


def embedding(tokens, table, scale):
    out = torch.zeros((*tokens.shape, table.shape[1]), dtype=torch.float64)
    ok = (tokens >= 0) & (tokens < table.shape[0])
    out[ok] = table.double()[tokens[ok].long()] * scale
    return out


def embedding_grad(tokens, dout, vocab, scale):
    """(gradient, sum of the absolute values of its terms, number of terms)."""
    d = dout.shape[-1]
    t, x = tokens.reshape(-1).long(), dout.reshape(-1, d).double()
    ok = (t >= 0) & (t < vocab)
    g = torch.zeros((vocab, d), dtype=torch.float64)
    s, c = torch.zeros_like(g), torch.zeros(vocab, dtype=torch.float64)
    g.index_add_(0, t[ok], x[ok])
    s.index_add_(0, t[ok], x[ok].abs())
    c.index_add_(0, t[ok], torch.ones(int(ok.sum()), dtype=torch.float64))
    return g * scale, s * abs(scale), c


def kept(x, group=32):
    """(q, exponents) of an 8-bit checkpoint of x [n, d], element by element."""
    n, d = x.shape
    y = x.double()
    q = torch.zeros((n, d), dtype=torch.int64)
    exps = torch.zeros((n, (d + group - 1) // group), dtype=torch.int64)
    for r in range(n):
        for c in range(exps.shape[1]):
            s = slice(c * group, min(d, (c + 1) * group))
            row = y[r, s]
            if not torch.isfinite(row).all():
                exps[r, c] = 255
                continue
            top, e = float(row.abs().max()), -126
            while _round_even(top / 2.0 ** e) > 127:
                e += 1
            if e > 121:  # 64 * 2^122 is no float
                e = 121
            exps[r, c] = e + 127
            q[r, s] = torch.tensor([max(-127, min(127, _round_even(float(t) / 2.0 ** e))) for t in row])
    return q, exps


def _round_even(t):
    return int(round(t))  # (Python rounds ties to even)


def unkept(q, exps, group=32):
    e = exps.repeat_interleave(group, 1)[:, :q.shape[1]].double()
    return torch.where(e == 255, math.nan, q.double() * torch.exp2(e - 127))


def act(x, name):
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x / math.sqrt(2)))
    return x / (1 + torch.exp(-1.702 * x)) if name == "quick_gelu" else x


def act_slope(x, name):
    if name == "gelu":
        return 0.5 * (1 + torch.erf(x / math.sqrt(2))) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-1.702 * x))
    return s * (1 + 1.702 * x * (1 - s))
