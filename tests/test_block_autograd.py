"""The block operators' autograd functions as the graph sees them, without a GPU (the
kernels' places are taken by torch products that leave no graph), and captured into a
HIP graph on one."""

import pytest
import torch

import paper_2410_17243_amd as infcl
from oracle import block as oracle
from paper_2410_17243_amd import block


@pytest.fixture
def plain_kernels(monkeypatch):
    """Stand-ins that compute on the CPU."""
    def turn(x, pos, freqs, sections=None, turned=None, paired="halves", back=False):
        y = oracle.turned(x.detach(), pos[:, None], freqs, (freqs.numel(),), x.shape[1] if turned is None else turned,
                          paired == "neighbours", back)[0]
        return y.to(x.dtype)

    def norm_fwd(x, y=None, gate=None, post_w=None, post_b=None, pre_w=None, pre_b=None, norm="layer", eps=1e-5, alpha=1.0,
                 p=0.0, seed=0, site=0, row0=0, need_grad=True):
        v = (gate, post_w, post_b, pre_w, pre_b)
        t = [None if a is None else a.detach() for a in (x, y, *v)]
        r = oracle.add_norm(*t, rms=norm == "rms", eps=eps, alpha=alpha)
        h, z = r.get("h"), r.get("z")
        return (x if h is None else h.to(x.dtype), None if z is None else z.to(x.dtype),
                infcl.AddNormKept(x, y, v, torch.zeros((x.numel() // x.shape[-1], 4)), (norm, eps, alpha, p, seed, site, row0)))

    def norm_bwd(dh, dz, kept, need=(True,) * 7):
        t = [None if a is None else a.detach() for a in (kept.x, kept.y, *kept.vectors, dh, dz)]
        r = oracle.add_norm(*t[:7], rms=kept.options[0] == "rms", eps=kept.options[1], alpha=kept.options[2], dh=t[7], dz=t[8])
        args = (kept.x, kept.y, *kept.vectors)
        return tuple(None if a is None or not n else r["d" + k].to(a.dtype) for a, n, k in
                     zip(args, need, ("x", "y", "gate", "post_w", "post_b", "pre_w", "pre_b")))

    def lin_fwd(x, w, b=None, need_dx=True, need_dw=True):
        y = torch.nn.functional.linear(x.detach(), w.detach(), None if b is None else b.detach())
        return y, (torch.cat([x.detach(), w.detach()]), (x.shape[0], need_dx, need_dw, b is not None))

    def lin_bwd(dy, kept, need=(True, True, True)):
        both, (n, need_dx, need_dw, has_b) = kept
        d = dy.detach()
        return (d @ both[n:] if need[0] and need_dx else None, d.t() @ both[:n] if need[1] and need_dw else None,
                d.sum(0) if need[2] and has_b else None)

    for name, fn in {
        "rotary_fwd": turn, "rotary_bwd": lambda d, *a: turn(d, *a, back=True),
        "dropout_fwd": lambda x, p, *a: x.detach() * oracle.kept(*x.shape, p, *a).to(x.dtype),
        "dropout_bwd": lambda x, p, *a: x.detach() * oracle.kept(*x.shape, p, *a).to(x.dtype),
        "add_norm_fwd": norm_fwd, "add_norm_bwd": norm_bwd, "linear_fp8_fwd": lin_fwd, "linear_fp8_bwd": lin_bwd,
    }.items():
        monkeypatch.setattr(block, name, fn)


def _call(name):
    """(the function of its differentiable arguments, those arguments)."""
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64).requires_grad_()  # noqa: E731
    pos, freqs = torch.tensor([0, 5, 9]), torch.tensor([1.0, 0.3, 0.1])
    both = lambda *a: torch.cat([t for t in infcl.add_norm(*a, alpha=0.5) if t is not None])  # noqa: E731
    return {
        "rotary": (lambda x: infcl.rotary(x, pos, freqs, turned=1), [r(3, 2, 8)]),
        "dropout": (lambda x: infcl.dropout(x, 0.25, 7, 2), [r(6, 8)]),
        "add_norm": (both, [r(6, 8), r(6, 8), r(8), r(8), r(8), r(8), r(8)]),
        "add_norm, no z": (both, [r(6, 8), r(6, 8), r(8)]),
        "add_norm, no y": (lambda x, w, b: infcl.add_norm(x, pre_w=w, pre_b=b, norm="rms")[1], [r(6, 8), r(8), r(8)]),
        "linear_fp8": (infcl.linear_fp8, [r(6, 8), r(16, 8), r(16)]),
    }[name]


NAMES = ["rotary", "dropout", "add_norm", "add_norm, no z", "add_norm, no y", "linear_fp8"]


@pytest.mark.parametrize("name", NAMES)
def test_gradients_by_differences(plain_kernels, name):
    f, args = _call(name)
    d = torch.randn(f(*args).shape, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    got = torch.autograd.grad((f(*args) * d).sum(), args)
    for i, a in enumerate(args):
        for at in range(0, a.numel(), 5):
            e = torch.zeros_like(a).detach()
            e.view(-1)[at] = 1e-6
            hi, lo = (float((f(*[t.detach() + s * e if j == i else t.detach() for j, t in enumerate(args)]) * d).sum()) for s in (1, -1))
            assert abs((hi - lo) / 2e-6 - float(got[i].reshape(-1)[at])) < 1e-6, (i, at)


@pytest.mark.parametrize("name", NAMES)
def test_second_derivatives_are_refused(plain_kernels, name):
    f, args = _call(name)
    first = torch.autograd.grad(f(*args).square().sum(), args, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (args[0].square().sum() + sum(x.square().sum() for x in first)).backward()


@pytest.mark.parametrize("name", NAMES)
def test_only_what_is_asked_for_has_a_gradient(plain_kernels, name):
    f, args = _call(name)
    full = torch.autograd.grad(f(*args).sum(), args)
    for i in range(len(args)):
        some = [a.detach().requires_grad_(j == i) for j, a in enumerate(args)]
        f(*some).sum().backward()
        assert torch.equal(some[i].grad, full[i]) and all(a.grad is None for j, a in enumerate(some) if j != i)


def _opaque(fn):
    """fn as a kernel is to torch: what it computes is not seen as torch operations."""
    def call(*args, **kw):
        plain = lambda t: torch.from_numpy(t.detach().numpy().copy()) if isinstance(t, torch.Tensor) and t.is_floating_point() else t  # noqa: E731
        res = fn(*(plain(a) for a in args), **{k: plain(a) for k, a in kw.items()})
        return plain(res) if isinstance(res, torch.Tensor) else tuple(plain(r) for r in res)
    return call


@pytest.fixture
def opaque_kernels(plain_kernels, monkeypatch):
    for name in ("rotary_fwd", "dropout_fwd", "add_norm_fwd", "linear_fp8_fwd"):
        monkeypatch.setattr(block, name, _opaque(getattr(block, name)))
    monkeypatch.setattr(block, "_times_packed", _opaque(lambda x, w, b: torch.nn.functional.linear(x, w.q.double(), b)))


def _apart(name):
    """_call with the arguments as tensors without gradients, and products of packed weights."""
    if name == "packed":
        g = torch.Generator().manual_seed(4)
        w = infcl.Fp8(torch.randint(0, 5, (16, 128), generator=g, dtype=torch.uint8), torch.full((16, 4), 127, dtype=torch.uint8), 128, torch.float64)
        return lambda x: infcl.linear_fp8(x, w), [torch.randn((3, 128), generator=g, dtype=torch.float64)]
    f, args = _call(name)
    return f, [a.detach() for a in args]


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("name", [*NAMES, "packed"])
def test_forward_mode_is_refused(opaque_kernels, name, grad):
    """A tensor that carries a tangent, and none that has gradients: no derivative is lost silently."""
    f, args = _apart(name)
    for i in range(len(args)):
        with torch.set_grad_enabled(grad), torch.autograd.forward_ad.dual_level():
            dual = [torch.autograd.forward_ad.make_dual(a, torch.ones_like(a)) if j == i else a for j, a in enumerate(args)]
            with pytest.raises(NotImplementedError):
                f(*dual)


@pytest.mark.parametrize("name", [*NAMES, "packed"])
def test_traced_calls_compute(opaque_kernels, name):
    """A trace of inputs without gradients holds the call, not one call's results."""
    f, args = _apart(name)
    traced = torch.jit.trace(f, tuple(args), check_trace=False)
    for seed in range(2):
        g = torch.Generator().manual_seed(seed)
        new = [torch.randn(a.shape, generator=g, dtype=a.dtype) for a in args]
        want = f(*new)
        assert torch.equal(traced(*new), want) and float(want.norm()) > 0
        with torch.no_grad():
            assert torch.equal(traced(*new), want)
        if name != "packed":  # (and its gradients, where they are asked for later)
            leaves = [a.requires_grad_() for a in new]
            assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(traced(*leaves).sum(), leaves),
                                                         torch.autograd.grad(f(*leaves).sum(), leaves)))


@pytest.mark.parametrize("name", ["dropout", "add_norm"])
def test_a_traced_seed_is_an_input(monkeypatch, name):
    """A seed in a tensor is read anew at every call of a trace."""
    seen = []
    monkeypatch.setattr(block, "dropout_fwd", lambda x, p, seed, *a: seen.append(int(seed)) or torch.zeros(x.shape))
    monkeypatch.setattr(block, "add_norm_fwd", lambda x, y, *v, seed, **k: seen.append(int(seed)) or (torch.zeros(x.shape), None, None))
    f = {"dropout": lambda x, s: infcl.dropout(x, 0.5, s), "add_norm": lambda x, s: infcl.add_norm(x, x, p=0.5, seed=s)[0]}[name]
    traced = torch.jit.trace(f, (torch.ones((6, 8)), torch.tensor([3])), check_trace=False)
    traced(torch.ones((6, 8)), torch.tensor([8]))
    assert seen == [3, 8]


@pytest.mark.gpu
def test_a_block_captured_into_a_graph():
    """Forward and backward of a run of all of them, captured once and replayed with new
    inputs and seeds between eager work: every replay gives what the eager calls give."""
    n, heads, hd, d, m = 300, 6, 32, 64, 192
    dt = torch.bfloat16
    r = lambda *s: torch.randn(s, device="cuda").to(dt)  # noqa: E731
    x, w, b, o, dq = r(n, d), r(m, d) / 8, r(m), r(d, m) / 14, r(n, heads, hd)
    gate, pw, dh, dz = r(d), r(d), r(n, d), r(n, d)
    pos, freqs = torch.arange(n, dtype=torch.int32, device="cuda"), infcl.rotary_freqs(16)
    seed = torch.tensor([5], device="cuda")

    def step():
        q, kept = infcl.linear_fp8_fwd(x, w, b)
        q = infcl.rotary_fwd(q.view(n, heads, hd), pos, freqs, turned=4)
        t, kept_o = infcl.linear_fp8_fwd(q.view(n, m), o)
        h, z, kept_n = infcl.add_norm_fwd(x, t, gate=gate, post_w=pw, pre_w=pw, norm="rms", p=0.2, seed=seed, site=1)
        z = infcl.dropout_fwd(z, 0.1, seed)
        dx, dt_, *dn = infcl.add_norm_bwd(dh, infcl.dropout_bwd(dz, 0.1, seed), kept_n)
        dt_, do, _ = infcl.linear_fp8_bwd(dt_, kept_o)
        dt_ = infcl.rotary_bwd(dt_.view(n, heads, hd), pos, freqs, turned=4)
        return [h, z, dx, *[t for t in dn if t is not None], do, *infcl.linear_fp8_bwd(dt_.view(n, m), kept)]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    seen = []
    for rep in range(4):
        x.copy_(r(n, d))
        seed.fill_(rep)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want)), rep
        seen.append(got[0])
    assert not torch.equal(seen[0], seen[1])


@pytest.mark.gpu
def test_on_a_stream_of_its_own():
    """Calls on another stream than the default one follow that stream's work."""
    x, w = torch.randn((2000, 512), device="cuda"), torch.randn(512, device="cuda")
    want = infcl.add_norm_fwd(x * 3, x, pre_w=w)[1]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y = x.clone()
        for _ in range(20):
            y = y * 1.0
        z = infcl.add_norm_fwd(y * 3, y, pre_w=w)[1]
    s.synchronize()
    assert torch.equal(z, want)


@pytest.mark.gpu
def test_runs_repeat_bit_for_bit():
    x, y, w = torch.randn((3001, 264), device="cuda").bfloat16(), torch.randn((3001, 264), device="cuda").bfloat16(), torch.randn(264, device="cuda")
    lw = torch.randn((520, 264), device="cuda").bfloat16()
    dy = torch.randn((3001, 520), device="cuda").bfloat16()

    def once():
        h, z, kept = infcl.add_norm_fwd(x, y, gate=w, pre_w=w, p=0.1, seed=1)
        o, k = infcl.linear_fp8_fwd(z, lw)
        return [h, z, o, *infcl.add_norm_bwd(h, z, kept), *infcl.linear_fp8_bwd(dy, k)]

    first = once()
    for _ in range(3):
        assert all(a is None or torch.equal(a, b) for a, b in zip(once(), first))


def _learn(x, w, b, o, gate, n, pos, freqs, seed):
    """A run of the differentiable calls, and its gradients."""
    q = infcl.rotary(infcl.linear_fp8(x, w, b).view(-1, 6, 32), pos, freqs, turned=4)
    t = infcl.dropout(infcl.linear_fp8(q.reshape(-1, 192), o), 0.1, seed)
    h, z = infcl.add_norm(x, t, gate, pre_w=n, p=0.2, seed=seed, site=1)
    return [h.detach(), z.detach(), *torch.autograd.grad((h * z).float().sum(), (x, w, b, o, gate, n))]


def _leaves(rows):
    r = lambda *s: torch.randn(s, device="cuda").bfloat16().requires_grad_()  # noqa: E731
    return [r(rows, 64), r(192, 64), r(192), r(64, 192), r(64), r(64)]


@pytest.mark.gpu
def test_a_step_with_autograd_captured_into_a_graph():
    """The differentiable calls and their gradients in a graph (no eager graph of the leaves
    is alive while it is captured): replays with new inputs and seeds, between eager work."""
    args = _leaves(300)
    pos, freqs, seed = torch.arange(300, dtype=torch.int32, device="cuda"), infcl.rotary_freqs(16), torch.tensor([5], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _learn(*args, pos, freqs, seed)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = _learn(*args, pos, freqs, seed)
    for rep in range(4):
        with torch.no_grad():
            args[0].copy_(torch.randn(300, 64, device="cuda"))
        seed.fill_(rep)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = _learn(*args, pos, freqs, seed)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want)), rep


@pytest.mark.gpu
def test_two_streams_at_once():
    """Calls on two streams share nothing: the results of each alone."""
    freqs, seed = infcl.rotary_freqs(16), torch.tensor([3], device="cuda")
    sets = [(_leaves(n), torch.arange(n, dtype=torch.int32, device="cuda")) for n in (2000, 1777)]
    want = [_learn(*a, pos, freqs, seed) for a, pos in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(5):
        for i, (a, pos) in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                got[i].append(_learn(*a, pos, freqs, seed))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, c) for a, c in zip(g, want[i]))


@pytest.mark.gpu
def test_a_trace_of_a_run():
    """torch.jit.trace of inputs without gradients: other inputs, and leaves, go through the
    kernels.  A tangent is refused."""
    args = [a.detach() for a in _leaves(40)]
    pos, freqs, seed = torch.arange(40, dtype=torch.int32, device="cuda"), infcl.rotary_freqs(16), torch.tensor([5], device="cuda")
    packed = infcl.fp8_pack(torch.randn((24, 64), device="cuda").bfloat16())

    def run(x, w, b, o, gate, n, seed):
        q = infcl.rotary(infcl.linear_fp8(x, w, b).view(-1, 6, 32), pos, freqs, turned=4)
        t = infcl.dropout(infcl.linear_fp8(q.reshape(-1, 192), o), 0.1, seed)
        return infcl.add_norm(x, t, gate, pre_w=n, p=0.2, seed=seed, site=1)

    traced = torch.jit.trace(run, (*args, seed), check_trace=False)
    last = torch.jit.trace(lambda x: infcl.linear_fp8(x, packed), (args[0],), check_trace=False)
    for rep in range(2):
        leaves, seed = _leaves(40), torch.tensor([rep], device="cuda")
        want, got = run(*leaves, seed), traced(*leaves, seed)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        grads = [torch.autograd.grad((h * z).float().sum(), leaves) for h, z in (want, got)]
        assert all(torch.equal(a, b) for a, b in zip(*grads))
        with torch.no_grad():
            assert all(torch.equal(a, b) for a, b in zip(traced(*leaves, seed), want))
            assert torch.equal(last(leaves[0]), infcl.linear_fp8(leaves[0], packed))
    with torch.no_grad(), torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(args[0], torch.ones_like(args[0]))
        for f in (lambda: infcl.dropout(dual, 0.1, 3), lambda: infcl.add_norm(dual, pre_w=args[5]), lambda: infcl.linear_fp8(dual, packed),
                  lambda: infcl.linear_fp8(dual, args[1]), lambda: infcl.rotary(dual.view(40, 2, 32), pos, freqs)):
            with pytest.raises(NotImplementedError):
                f()
