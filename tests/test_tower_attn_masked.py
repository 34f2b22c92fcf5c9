"""What masked rows hold reaches no one, and what that costs: sweeps whose tiles a
causal mask cuts, with entries that are not finite in rows that some own rows see and
some do not, in every form of the kernels (one wave or four, sweeps in parts, shared
heads, lengths longer than said)."""

import ctypes
import math

import pytest
import torch

import paper_2410_17243_amd as infcl
from oracle import tower
from paper_2410_17243_amd import tower as binding

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # one rounding to nearest
F32 = 2.0 ** -15  # (scores off by less than 2^-17, exponentials and sums of fp32)
TINY = {"bf16": 1e-30, "f16": 2.0 ** -25}

# lengths, heads, kv heads, head_dim, type, said longest length, parts of the sweeps
# over queries and over keys of the backward pass
CASES = [
    ([20, 45], 2, 2, 64, "f16", 45, 1, 1),
    ([31, 7], 4, 1, 128, "bf16", 31, 1, 1),          # 124 rows, one wave
    ([150, 300], 2, 1, 64, "bf16", 300, 1, 1),
    ([700], 3, 3, 64, "f16", 700, 1, 2),
    ([520, 300], 4, 1, 128, "bf16", 520, 4, 2),
    ([520, 300], 4, 1, 80, "f16", 520, 4, 2),
    ([1100, 400], 4, 2, 64, "f16", 1100, 4, 4),
    ([1100, 400], 4, 2, 64, "bf16", 600, 2, 2),      # longer than said
]


def _cu(lens):
    return [0] + torch.tensor(lens).cumsum(0).tolist()


def _inputs(lens, heads, kv, hd, dtype):
    g = torch.Generator().manual_seed(sum(lens))
    t = sum(lens)
    return [torch.randn((t, h, hd), generator=g).to(DT[dtype]) for h in (heads, kv, kv, heads)]


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda") if isinstance(x, list) else x.cuda()


@pytest.mark.parametrize("lens,heads,kv,hd,dtype,said,parts,parts_q", CASES)
def test_the_cases_are_cut_as_they_say(lens, heads, kv, hd, dtype, said, parts, parts_q):
    up = lambda x: (x + 255) // 256 * 256  # noqa: E731
    t = sum(lens)
    shape = binding._Shape(t, t, len(lens), heads, kv, hd, binding._CODES[DT[dtype]], 1, said, said, hd ** -0.5)
    b = ctypes.c_size_t(0)
    assert binding._load().infcl_attn_workspace(ctypes.byref(shape), None, ctypes.byref(b)) == 0
    stat = up(2 * ((t + 32 + 63) // 64 * 64) * heads * 4)
    dkv = 2 * parts * t * kv * hd * 4 if parts > 1 else 0
    dq = parts_q * t * heads * hd * 4 if parts_q > 1 else 0
    assert b.value == up(stat + max(dkv, dq))


def _tol(r, name, e, dtype):
    t = (e + F32) * r[name + "_abs"] + e * r[name].abs() + TINY[dtype]
    return t + (e + F32) * r[name + "_dlt"] if name in ("dq", "dk") else t


def _near(got, want, tol, what):
    got = got.cpu().double()
    assert torch.isfinite(got).all(), what
    assert ((got - want).abs() <= tol).all(), (what, float(((got - want).abs() - tol).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("lens,heads,kv,hd,dtype,said,parts,parts_q", CASES)
def test_an_entry_reaches_those_who_see_it(lens, heads, kv, hd, dtype, said, parts, parts_q, bad):
    """One entry of one row of the last sequence is not finite, in a tile that the mask
    cuts.  Every other value is that of the same inputs without it, element by
    element."""
    cu, e, g = _cu(lens), EPS[dtype], heads // kv
    q, k, v, do = _inputs(lens, heads, kv, hd, dtype)
    scale = hd ** -0.5
    r = tower.attention(q, k, v, cu, cu, True, scale, do)
    at, f = cu[-2] + lens[-1] * 2 // 5, hd - 3
    call = dict(cu_q=_dev(cu), max_q=said)
    a = [_dev(x) for x in (q, k, v, do)]
    out, lse = infcl.packed_attn_fwd(*a[:3], **call)

    def with_bad(x, head):
        y = x.clone()
        y[at, head, f] = bad
        return y

    # a value: feature f of the queries that see it, and no other element
    got = infcl.packed_attn_fwd(a[0], a[1], with_bad(a[2], kv - 1), **call)[0]
    mask = torch.zeros((sum(lens), heads, hd), dtype=torch.bool)
    mask[at:, (kv - 1) * g:, f] = True
    assert not torch.isfinite(got.cpu()[mask]).any()
    if bad == bad:
        assert (got.cpu()[mask] == bad).all()
    clean = torch.where(mask, 0.0, got.cpu().double())
    _near(clean, torch.where(mask, 0.0, r["out"]), _tol(r, "out", e, dtype), "out")
    # a key (of unit scores without it, as the statistics come from there): dq of the queries that see it
    dq = infcl.packed_attn_bwd(a[0], with_bad(a[1], kv - 1), a[2], out, lse, a[3], **call)[0].cpu()
    mask = torch.zeros((sum(lens), heads, hd), dtype=torch.bool)
    mask[at:, (kv - 1) * g:] = True
    assert not torch.isfinite(dq[at:, (kv - 1) * g:, f]).any()
    _near(torch.where(mask, 0.0, dq.double()), torch.where(mask, 0.0, r["dq"]), _tol(r, "dq", e, dtype), "dq")
    # dout of one query and head: its own dq, dk of the keys it sees, feature f of their dv
    dq, dk, dv = [x.cpu() for x in infcl.packed_attn_bwd(*a[:3], out, lse, with_bad(a[3], heads - 1), **call)]
    mine = torch.zeros((sum(lens), kv, hd), dtype=torch.bool)
    mine[cu[-2]:at + 1, kv - 1] = True
    assert not torch.isfinite(dk[mine]).any()
    _near(torch.where(mine, 0.0, dk.double()), torch.where(mine, 0.0, r["dk"]), _tol(r, "dk", e, dtype), "dk")
    mine[:, :, :f], mine[:, :, f + 1:] = False, False
    assert not torch.isfinite(dv[mine]).any()
    _near(torch.where(mine, 0.0, dv.double()), torch.where(mine, 0.0, r["dv"]), _tol(r, "dv", e, dtype), "dv")
    assert not torch.isfinite(dq[at, heads - 1]).any()
    dq[at, heads - 1] = r["dq"][at, heads - 1].to(dq.dtype)
    _near(dq, r["dq"], _tol(r, "dq", e, dtype), "dq")


@pytest.mark.gpu
@pytest.mark.parametrize("lens,heads,kv,hd,dtype,said,parts,parts_q", CASES)
def test_rows_that_only_some_see_hold_nothing_finite(lens, heads, kv, hd, dtype, said, parts, parts_q):
    """The last sequence's second half is all NaN or infinities, on the side that the
    first half does not see; and its first half, on the side that the second
    half's keys are not seen by."""
    cu, e = _cu(lens), EPS[dtype]
    q, k, v, do = _inputs(lens, heads, kv, hd, dtype)
    r = tower.attention(q, k, v, cu, cu, True, hd ** -0.5, do)
    at = cu[-2] + lens[-1] // 2
    call = dict(cu_q=_dev(cu), max_q=said)
    a = [_dev(x) for x in (q, k, v, do)]
    out, lse = infcl.packed_attn_fwd(*a[:3], **call)
    bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda", dtype=DT[dtype])

    def spoil(x, s):
        y = x.clone()
        y[s] = bad[torch.arange(y[s].numel(), device="cuda") % 3].view(y[s].shape)
        return y

    late, early = slice(at, None), slice(cu[-2], at)
    k2, v2 = spoil(a[1], late), spoil(a[2], late)
    got, got_lse = infcl.packed_attn_fwd(a[0], k2, v2, **call)
    _near(got[:at], r["out"][:at], _tol(r, "out", e, dtype)[:at], "out")
    assert ((got_lse[:, :at].cpu().double() - r["lse"][:, :at]).abs() <= 2.0 ** -16 + 2.0 ** -22 * r["lse"][:, :at].abs()).all()
    assert not torch.isfinite(got[late]).any()
    dq = infcl.packed_attn_bwd(a[0], k2, v2, out, lse, a[3], **call)[0]
    _near(dq[:at], r["dq"][:at], _tol(r, "dq", e, dtype)[:at], "dq")
    _, dk, dv = infcl.packed_attn_bwd(spoil(a[0], early), a[1], a[2], out, lse, spoil(a[3], early), **call)
    _near(dk[at:], r["dk"][at:], _tol(r, "dk", e, dtype)[at:], "dk")
    _near(dv[at:], r["dv"][at:], _tol(r, "dv", e, dtype)[at:], "dv")
    assert not torch.isfinite(dk[early]).any() and not torch.isfinite(dv[early]).any()


@pytest.mark.gpu
def test_a_step_that_overflowed_takes_about_as_long():
    """fp16 with loss scaling overflows now and then: one infinite row of dout that
    every key of its sequence is seen by, and a dout of nothing but NaN.  (The rows
    that mask-cut tiles hold are taken one by one: measured 5 and 8 times a clean step's
    time.  The bound leaves room for a busy machine; a sweep of all rows one by one
    is past a thousand.)"""
    n, length = 2, 2048
    g = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda h: torch.randn((n * length, h, 128), generator=g, device="cuda").half()  # noqa: E731
    q, k, v, do = mk(8), mk(2), mk(2), mk(8)
    cu = _dev([0, length, 2 * length])
    out, lse = infcl.packed_attn_fwd(q, k, v, cu, length)

    def time(d):
        took = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            infcl.packed_attn_bwd(q, k, v, out, lse, d, cu, length)
            b.record()
            torch.cuda.synchronize()
            took.append(a.elapsed_time(b))
        return min(took)

    clean, one = time(do), do.clone()
    one[length // 2] = math.inf
    assert time(one) < 100 * clean and time(torch.full_like(do, math.nan)) < 100 * clean


@pytest.mark.gpu
@pytest.mark.parametrize("n,heads,kv,hd", [(5, 2, 1, 64), (200, 2, 2, 128), (3000, 4, 1, 64)])
def test_scores_of_minus_infinity(n, heads, kv, hd):
    """Keys whose scores are all -infinity weigh nothing beside others; a query that
    sees no others has no weights at all: NaN, not the zeros of a query that sees no
    key."""
    g = torch.Generator().manual_seed(n)
    q, k, v = (torch.rand((n, h, hd), generator=g).bfloat16() + 0.5 for h in (heads, kv, kv))
    k[:n // 3] = -math.inf  # (q is positive)
    a, cu = [x.cuda() for x in (q, k, v)], _dev([0, n])
    first = n // 3
    out, lse = infcl.packed_attn_fwd(*a, cu, n)
    assert torch.isnan(out[:first]).all() and torch.isnan(lse[:, :first]).all()
    r = tower.attention(q[first:], k[first:], v[first:], [0, n - first], [0, n - first], True, hd ** -0.5)
    _near(out[first:], r["out"], _tol(r, "out", EPS["bf16"], "bf16"), "out")
    # one query over all the keys (in parts where there are many), over the first third, over none
    for keys, want in ((n, 0), (first, math.nan), (0, 0)):
        one, lse = infcl.packed_attn_fwd(a[0][-1:], a[1], a[2], _dev([0, 1]), 1, _dev([0, keys]), keys)
        if want != want:
            assert torch.isnan(one).all() and torch.isnan(lse).all()
        elif keys:
            assert (one[0].double() - out[-1].double()).abs().max() <= 4 * EPS["bf16"] * 1.5
        else:
            assert (one == 0).all() and (lse == -math.inf).all()
