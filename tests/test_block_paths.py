"""Forms of the block operators' kernels that the host chooses by size, and addresses past
32 bits."""

import pytest
import torch

import paper_2410_17243_amd as infcl

FAR = 32 << 20  # outputs above this many bytes are stored past the caches


@pytest.mark.gpu
def test_large_outputs_are_those_of_their_parts():
    """Rows of outputs above 32 MB, which leave past the caches, bit for bit those of calls
    below that."""
    n, d = 9001, 2048
    assert n * d * 2 > FAR > (n // 2 + 1) * d * 2
    x, y = (torch.randn((n, d), device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(d, device="cuda")
    cut = [(0, n // 2), (n // 2, n)]
    whole = infcl.dropout_fwd(x, 0.3, 5, site=2)
    assert torch.equal(whole, torch.cat([infcl.dropout_fwd(x[a:b], 0.3, 5, site=2, row0=a) for a, b in cut]))
    pos, freqs = torch.arange(n, dtype=torch.int32, device="cuda"), infcl.rotary_freqs(64)
    for paired, pairs in (("halves", 64), ("halves", 61), ("neighbours", 60)):
        f = freqs[:pairs].contiguous()
        turn = lambda a, b: infcl.rotary_fwd(x[a:b].view(-1, 16, 128), pos[a:b], f, None, 12, paired)  # noqa: E731
        assert torch.equal(turn(0, n), torch.cat([turn(a, b) for a, b in cut]))
    for kw in (dict(pre_w=w), dict(pre_w=w, gate=w, post_w=w, p=0.1, seed=3), dict(pre_w=w, post_w=w, post_b=w)):
        whole = infcl.add_norm_fwd(x, y, **kw)
        parts = [infcl.add_norm_fwd(x[a:b], y[a:b], row0=a, **kw) for a, b in cut]
        for i in range(2):
            assert torch.equal(whole[i], torch.cat([p[i] for p in parts]))
        grads = infcl.add_norm_bwd(x, y, whole[2])
        some = [infcl.add_norm_bwd(x[a:b], y[a:b], p[2]) for (a, b), p in zip(cut, parts)]
        for i in range(2):
            assert torch.equal(grads[i], torch.cat([s[i] for s in some]))


def _wide(n, d, dtype, stride):
    """n rows of d entries, `stride` entries apart."""
    return torch.empty((n - 1) * stride + d, dtype=dtype, device="cuda").as_strided((n, d), (stride, 1))


@pytest.mark.gpu
def test_rows_more_than_2_gib_apart():
    """Offsets past 31 and 32 bits, in entries and bytes."""
    n, d, stride = 4, 64, 1 << 30
    x, y = torch.randn((n, d), device="cuda").bfloat16(), torch.randn((n, d), device="cuda").bfloat16()
    far = _wide(n, d, torch.bfloat16, stride)
    far.copy_(x)
    w = torch.randn(d, device="cuda")
    assert torch.equal(infcl.dropout_fwd(far, 0.5, 1), infcl.dropout_fwd(x, 0.5, 1))
    a, b = infcl.add_norm_fwd(far, y, pre_w=w), infcl.add_norm_fwd(x, y, pre_w=w)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert all(s is t or torch.equal(s, t) for s, t in zip(infcl.add_norm_bwd(far, y, a[2]), infcl.add_norm_bwd(x, y, b[2])))
    pos, freqs = torch.arange(n, dtype=torch.int32, device="cuda"), infcl.rotary_freqs(16)
    assert torch.equal(infcl.rotary_fwd(far.view(n, 2, 32), pos, freqs), infcl.rotary_fwd(x.view(n, 2, 32), pos, freqs))
    p, q = infcl.fp8_pack_both(far), infcl.fp8_pack_both(x)
    assert all(torch.equal(s.q, t.q) and torch.equal(s.exps, t.exps) for s, t in zip(p, q))
    lw = infcl.fp8_pack(torch.randn((8, d), device="cuda").bfloat16())
    assert torch.equal(infcl.linear_fp8(far, lw), infcl.linear_fp8(x, lw))


@pytest.mark.gpu
def test_operands_of_more_than_4_gib():
    """The last rows of an operand of 4.5 GB, and of an output of 9 GB, are where they belong."""
    k, n = 65536, 72000
    x = torch.zeros((n, k), dtype=torch.int8, device="cuda")
    at = torch.arange(n, device="cuda")
    x[at, at % k] = (at % 7 + 1).to(torch.int8)
    p = infcl.fp8_pack(x[:8].bfloat16())
    q = torch.zeros((n, p.q.shape[1]), dtype=torch.uint8, device="cuda")
    e = torch.full((n, p.exps.shape[1]), 127, dtype=torch.uint8, device="cuda")
    for a in range(0, n, 8000):
        part = infcl.fp8_pack(x[a:a + 8000].bfloat16())
        q[a:a + 8000, :k], e[a:a + 8000] = part.q[:, :k], part.exps
    big = infcl.Fp8(q, e, k, torch.bfloat16)
    ones = infcl.fp8_pack(torch.ones((8, k), dtype=torch.bfloat16, device="cuda"))
    assert q.numel() > 1 << 32
    want = (at % 7 + 1).bfloat16()
    assert torch.equal(infcl.fp8_matmul(big, ones)[:, 3], want)
    assert torch.equal(infcl.fp8_matmul(ones, big)[5], want)
    del x, q, e, big
    a = infcl.fp8_pack(torch.ones((72000, 8), dtype=torch.bfloat16, device="cuda") * (at % 7 + 1).bfloat16()[:, None])
    b = infcl.fp8_pack(torch.eye(8, device="cuda").bfloat16().repeat(8192, 1))
    out = infcl.fp8_matmul(a, b)
    assert out.numel() > 1 << 32
    assert torch.equal(out[:, 65535], want) and torch.equal(out[71999], want[71999].expand(65536))


@pytest.mark.gpu
def test_the_longest_contraction():
    """2^23 entries: whole numbers, whose sums fp32 holds."""
    k = 1 << 23
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = (torch.randint(-1, 2, (s, k), generator=g, device="cuda", dtype=torch.int8).bfloat16() for s in (3, 9))
    out = infcl.fp8_matmul(infcl.fp8_pack(x), infcl.fp8_pack(w))
    assert torch.equal(out, (x.float() @ w.float().t()).bfloat16())
    with pytest.raises(infcl.InfclError):
        infcl.fp8_pack(torch.empty((1, k + 8), dtype=torch.bfloat16, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 15, 16, 17, 31])
@pytest.mark.parametrize("k", [8, 128, 520, 4096, 4104, 9000])
def test_few_rows(n, k):
    """Up to 16 rows are packed on the way, in spans of 4096 entries: what the packed product
    gives of whole numbers, a bias and odd outputs with it."""
    g = torch.Generator().manual_seed(n * k)
    x, w = (torch.randint(-3, 4, (s, k), generator=g).bfloat16().cuda() for s in (n, 37))
    b = torch.randint(-9, 9, (37,), generator=g).bfloat16().cuda()
    packed = infcl.fp8_pack(w)
    out = infcl.linear_fp8(x, packed, b)
    assert torch.equal(out, infcl.fp8_matmul(infcl.fp8_pack(x), packed, b))
    assert torch.equal(out, (x.double() @ w.double().t() + b.double()).bfloat16())
    odd = torch.zeros(38, dtype=torch.bfloat16, device="cuda")[1:].copy_(b)  # (begins at an odd entry)
    assert torch.equal(infcl.linear_fp8(x, packed, odd), out)
