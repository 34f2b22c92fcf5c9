"""Timed cases of the text tower's operators: what a program that trains or runs
an encoder beside the contrastive loss asks of them.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges,
``prepare`` makes one case's inputs on the GPU, ``run`` is one pass: through the
public entry points where ``own`` is true, else in elementary fp32 torch
operations.  ``exact`` is the same from the definitions in fp64.

Kinds of call (a case's "kind"):
  attn_train   packed attention, forward and backward: one layer of a training
               step over samples of different lengths
  attn_fwd     its forward with the log-sum-exp: embedding a held-out set
  attn_token   one query token per sequence over the keys so far: a prompt that
               is extended token by token
  embed        token embedding, forward and the table's gradient
  linear8      a layer's input kept in 8 bits and the layer's weight gradient
               from it (optionally through the activation)
  act8         an activation whose input is kept in 8 bits, and its backward
               from them

Attention entries are of unit size, as after a projection with unit gain, so
that the scores of scale 1/sqrt(head_dim) are of unit size too.  Caption lengths
are lognormal; other lengths are uniform up to the case's bound.  Token ids are
Zipf-like, with the first and the last id opening and closing every caption.
Activations have a few large features, as those of trained encoders do.
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GROUP = 32  # features that share a scale in 8-bit checkpoints


def _attn(kind, n, most, heads, kv, hd, dtype, causal=True, lens="uniform", fused=False, lens_seed=1):
    return {"kind": kind, "n": n, "most": most, "heads": heads, "kv": kv, "hd": hd, "dtype": dtype, "causal": causal,
            "lens": lens, "fused": fused, "lens_seed": lens_seed}


def _embed(n, vocab, d, dtype, ids="i64", scale=1.0):
    return {"kind": "embed", "n": n, "vocab": vocab, "d": d, "dtype": dtype, "ids": ids, "scale": scale}


def _linear8(n, d, m, dtype, act="none", grad="f32"):
    return {"kind": "linear8", "n": n, "d": d, "m": m, "dtype": dtype, "act": act, "grad": grad}


def _act8(n, d, dtype, act):
    return {"kind": "act8", "n": n, "d": d, "dtype": dtype, "act": act}


def listed():
    return [
        # one layer over a chunk of captions of a width-512 text tower, q, k, v views of one projection
        dict(_attn("attn_train", 1024, 77, 8, 8, 64, "bf16", lens="captions", fused=True), name="train_captions_1024"),
        # long documents with grouped heads: where the products count
        dict(_attn("attn_train", 4, 4096, 16, 4, 128, "bf16"), name="train_long_grouped_4x4096"),
        # a few samples of odd sizes in half precision, heads of 80 features, every token sees all
        dict(_attn("attn_train", 37, 301, 10, 5, 80, "f16", causal=False), name="train_full_odd_hd80"),
        # image patches of a held-out set, every token sees all
        dict(_attn("attn_fwd", 256, 257, 16, 16, 64, "f16", causal=False, lens="equal"), name="fwd_patches_256x257"),
        # the smallest call: one prompt's next token
        dict(_attn("attn_token", 1, 777, 8, 8, 64, "bf16", lens="equal"), name="token_1x777"),
        # many long prompts' next tokens with grouped heads: the keys' bytes
        dict(_attn("attn_token", 64, 8192, 32, 8, 128, "bf16"), name="token_64x8192_grouped"),
        # a micro-batch's tokens, fp32 table
        dict(_embed(2001, 8192, 512, "f32", ids="i32", scale=math.sqrt(512.0)), name="embed_2001_f32"),
        # the tokens of a batch of 32768 captions of about 16 tokens
        dict(_embed(524288, 50000, 512, "bf16"), name="embed_524288_bf16"),
        # a micro-batch through a layer of width 512
        dict(_linear8(2002, 512, 512, "bf16"), name="linear8_2002_512"),
        # a large chunk through the second layer of a block, the activation taken again from 8 bits
        dict(_linear8(65536, 4096, 1024, "bf16", act="gelu", grad="bf16"), name="linear8_65536_4096_gelu"),
        # a chunk through an odd-sized layer in half precision
        dict(_linear8(10007, 776, 1000, "f16"), name="linear8_10007_776_f16"),
        # the activation of that large chunk
        dict(_act8(65536, 4096, "bf16", "gelu"), name="act8_65536_4096"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _odd(rng, lo, hi):
    return min(_log(rng, lo, hi) | 1, hi)


def _width(rng):
    """A power of two from 32 to 4096, or an odd multiple of 8 in between."""
    return rng.choice([2 ** rng.randrange(5, 13), 8 * (_log(rng, 4, 511) | 1)])


def draw(rng):
    kind = rng.choice(["attn_train", "attn_train", "attn_fwd", "attn_token", "embed", "linear8", "act8"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    hd = rng.choice([32, 64, 64, 72, 80, 96, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 1, 2, 3, 4, 8])
    if kind in ("attn_train", "attn_fwd"):
        # the longest, most heads and most sequences not at once: at most half the scores of the largest listed.  A
        # training step has something to learn from two keys on (the gradients of q and k are zero with one)
        while True:
            most, n = _odd(rng, 2 if kind == "attn_train" else 1, 4096), _odd(rng, 1, 1024)
            if n * most * most * kv * group <= 2 ** 28 and n * most * kv * group * hd <= 2 ** 26:
                break
        lens = "captions" if most <= 128 and rng.random() < 0.5 else rng.choice(["uniform", "uniform", "equal"])
        return _attn(kind, n, most, kv * group, kv, hd, dtype, rng.random() < 0.7, lens,
                     rng.random() < 0.5, rng.randrange(1 << 16))
    if kind == "attn_token":
        while True:
            most, n = _odd(rng, 1, 16384), _odd(rng, 1, 256)
            if n * most * kv * hd <= 2 ** 28:
                break
        return _attn(kind, n, most, kv * group, kv, hd, dtype, True, "uniform", False,
                     rng.randrange(1 << 16))
    if kind == "embed":
        dtype = rng.choice(["bf16", "f16", "f32"])
        d = 8 * _log(rng, 4, 128)
        n = _odd(rng, 1, min(524288, (1 << 28) // d))
        return _embed(n, _odd(rng, 100, 100000), d, dtype, rng.choice(["i32", "i64"]), rng.choice([1.0, math.sqrt(d)]))
    if kind == "linear8":
        n, d, m = _odd(rng, 1, 65536), _width(rng), _width(rng)
        while n * d * m > 2 ** 38:
            n = n // 2 | 1
        act = rng.choice(["none", "none", "gelu", "quick_gelu"])
        return _linear8(n, d, m, dtype, act, "f32" if act == "none" else dtype)
    n, d = _odd(rng, 1, 65536), _width(rng)
    return _act8(n, d, rng.choice(["bf16", "f16", "f32"]) if n * d <= 2 ** 26 else dtype, rng.choice(["gelu", "quick_gelu"]))


# ------------------------------------------------------------------- inputs

def _lengths(case):
    """Key lengths of the case's sequences, from the case alone; one is the bound itself, one of many is empty."""
    rs = np.random.RandomState(case["lens_seed"])
    n, most = case["n"], case["most"]
    if case["lens"] == "equal":
        return np.full(n, most, dtype=np.int64)
    if case["lens"] == "captions":
        lens = np.clip(np.rint(np.exp(rs.normal(math.log(16.0), 0.5, n))), min(3, most), most).astype(np.int64)
    else:
        lens = rs.randint(1, most + 1, n).astype(np.int64)
    lens[rs.randint(n)] = most
    if n > 8:
        lens[np.argmin(lens)] = 0
    return lens


def _offsets(lens, dev):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).to(dev)


def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + salt)
    return g


def _normal(shape, dt, seed, salt):
    return torch.randn(shape, generator=_gen(seed, salt), device="cuda", dtype=torch.float32).to(dt)


def _activations(n, d, dt, seed, salt):
    """Rows of unit entries in which one feature of 64 is 8 times as large."""
    x = torch.randn((n, d), generator=_gen(seed, salt), device="cuda", dtype=torch.float32)
    gain = torch.where(torch.rand(d, generator=_gen(seed, salt + 1), device="cuda") < 1.0 / 64, 8.0, 1.0)
    return (x * gain).to(dt)


def prepare(case, seed):
    dt = DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"].startswith("attn"):
        lens = _lengths(case)
        token = case["kind"] == "attn_token"
        tk, heads, kv, hd = int(lens.sum()), case["heads"], case["kv"], case["hd"]
        tq = case["n"] if token else tk
        if case["fused"]:
            qkv = _normal((tk, heads + 2 * kv, hd), dt, seed, 1)
            st["q"], st["k"], st["v"] = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
        else:
            st["q"] = _normal((tq, heads, hd), dt, seed, 1)
            st["k"], st["v"] = _normal((tk, kv, hd), dt, seed, 2), _normal((tk, kv, hd), dt, seed, 3)
        st["cu_k"] = _offsets(lens, "cuda")
        st["cu_q"] = _offsets(np.ones(case["n"], np.int64), "cuda") if token else st["cu_k"]
        st["max_k"] = int(lens.max())
        st["max_q"] = 1 if token else st["max_k"]
        if case["kind"] == "attn_train":
            st["dout"] = _normal((tq, heads, hd), dt, seed, 4)
    elif case["kind"] == "embed":
        n, vocab = case["n"], case["vocab"]
        u = torch.rand(n, generator=_gen(seed, 5), device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)
        ids[::16] = 0
        ids[15::16] = vocab - 1
        st["tokens"] = ids.to(torch.int32) if case["ids"] == "i32" else ids
        st["table"] = (0.02 * _normal((vocab, case["d"]), torch.float32, seed, 6)).to(dt)
        st["dout"] = _normal((n, case["d"]), dt, seed, 7)
    elif case["kind"] == "linear8":
        st["x"] = _activations(case["n"], case["d"], dt, seed, 8)
        st["dy"] = _normal((case["n"], case["m"]), dt, seed, 10)
    else:
        st["x"] = _activations(case["n"], case["d"], dt, seed, 8)
        st["dy"] = _normal((case["n"], case["d"]), dt, seed, 10)
    return st


# ------------------------------------------------- one pass through the library

def _run_own(st):
    import paper_2410_17243_amd as infcl

    case = st["case"]
    kind = case["kind"]
    if kind == "attn_train":
        out, lse = infcl.packed_attn_fwd(st["q"], st["k"], st["v"], st["cu_q"], st["max_q"], causal=case["causal"])
        dq, dk, dv = infcl.packed_attn_bwd(st["q"], st["k"], st["v"], out, lse, st["dout"], st["cu_q"], st["max_q"],
                                           causal=case["causal"])
        return {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if kind == "attn_fwd":
        out, lse = infcl.packed_attn_fwd(st["q"], st["k"], st["v"], st["cu_q"], st["max_q"], causal=case["causal"])
        return {"out": out, "lse": lse}
    if kind == "attn_token":
        out, _ = infcl.packed_attn_fwd(st["q"], st["k"], st["v"], st["cu_q"], 1, st["cu_k"], st["max_k"],
                                       causal=case["causal"], need_lse=False)
        return {"out": out}
    if kind == "embed":
        out = infcl.embed_fwd(st["tokens"], st["table"], case["scale"])
        dtable = infcl.embed_bwd(st["tokens"], st["dout"], case["vocab"], case["scale"])
        return {"out": out, "dtable": dtable}
    if kind == "linear8":
        kept = infcl.ckpt8_pack(st["x"])
        return {"dw": infcl.ckpt8_wgrad(st["dy"], kept, act=case["act"], grad_dtype=DTYPES[case["grad"]])}
    out, kept = infcl.ckpt8_act_fwd(st["x"], case["act"])
    return {"out": out, "dx": infcl.ckpt8_act_bwd(st["dy"], kept, case["act"])}


# ------------------------------------------------------------ the plain forms

def _rows_of(x, cu, most):
    """Packed rows [t, heads, hd] as [n, heads, most, hd] in fp32; rows past a sequence's end are some other row's."""
    at = cu[:-1, None].long() + torch.arange(most, device=x.device)
    return x[at.clamp(max=max(x.shape[0] - 1, 0))].float().transpose(1, 2)


def _packed(x, cu, t):
    """Back to packed rows: [n, heads, most, hd] -> [t, heads, hd]."""
    row = torch.arange(t, device=x.device)
    seq = torch.searchsorted(cu[1:].contiguous(), row.to(cu.dtype), right=True)
    return x.transpose(1, 2)[seq, row - cu[:-1].long()[seq]]


def _plain_attn(st):
    case = st["case"]
    q, k, v, cu_q, cu_k, mq, mk = (st[x] for x in ("q", "k", "v", "cu_q", "cu_k", "max_q", "max_k"))
    n, kv, hd = case["n"], case["kv"], case["hd"]
    group = case["heads"] // kv
    scale = 1.0 / math.sqrt(hd)
    dt = q.dtype
    grouped = (n, kv, group * mq, hd)
    whole = (n, kv * group, mq, hd)
    fq, fk, fv = _rows_of(q, cu_q, mq).reshape(grouped), _rows_of(k, cu_k, mk), _rows_of(v, cu_k, mk)
    lq, lk = (cu_q[1:] - cu_q[:-1]).view(n, 1, 1), (cu_k[1:] - cu_k[:-1]).view(n, 1, 1)
    i, j = torch.arange(mq, device=q.device).view(1, mq, 1), torch.arange(mk, device=q.device).view(1, 1, mk)
    seen = (j < lk) & (i < lq)
    if case["causal"]:
        seen = seen & (j <= i + lk - lq)
    seen = seen.view(n, 1, 1, mq, mk)
    s = (torch.matmul(fq, fk.transpose(-1, -2)) * scale).view(n, kv, group, mq, mk).masked_fill(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = torch.exp(s - top)
    z = p.sum(-1, keepdim=True)
    lse = torch.where(z > 0, top + torch.log(z), -math.inf)
    p = (p / torch.where(z > 0, z, 1.0)).view(n, kv, group * mq, mk)
    out = torch.matmul(p, fv)
    res = {"out": _packed(out.view(whole), cu_q, q.shape[0]).to(dt)}
    if case["kind"] == "attn_fwd":
        res["lse"] = _packed(lse.view(n, kv * group, mq, 1), cu_q, q.shape[0])[..., 0].t().contiguous()
    if case["kind"] == "attn_train":
        do = _rows_of(st["dout"], cu_q, mq).reshape(grouped)
        dv = torch.matmul(p.transpose(-1, -2), do)
        ds = p * (torch.matmul(do, fv.transpose(-1, -2)) - (do * out).sum(-1, keepdim=True))
        dq = torch.matmul(ds, fk) * scale
        dk = torch.matmul(ds.transpose(-1, -2), fq) * scale
        res["dq"] = _packed(dq.view(whole), cu_q, q.shape[0]).to(dt)
        res["dk"], res["dv"] = _packed(dk, cu_k, k.shape[0]).to(dt), _packed(dv, cu_k, k.shape[0]).to(dt)
    return res


def _plain_embed(st):
    case = st["case"]
    ids = st["tokens"].long()
    out = (st["table"].float()[ids] * case["scale"]).to(st["table"].dtype)
    dtable = torch.zeros((case["vocab"], case["d"]), dtype=torch.float32, device=ids.device)
    dtable.index_add_(0, ids, st["dout"].float())
    return {"out": out, "dtable": dtable * case["scale"]}


def _plain_kept(x):
    """What 8-bit checkpoints of x stand for: groups of 32 features, the least power of two that keeps |q| <= 127."""
    n, d = x.shape
    g = torch.nn.functional.pad(x.float(), (0, -d % GROUP)).view(n, -1, GROUP)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.frexp(top)[1] - 7
    e = (e + (torch.round(torch.ldexp(top, -e)) > 127)).clamp(min=-126)
    return torch.ldexp(torch.round(torch.ldexp(g, -e)), e).view(n, -1)[:, :d]


def _plain_act(x, act):
    if act == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if act == "quick_gelu":
        return x / (1.0 + torch.exp(-1.702 * x))
    return x


def _plain_act_slope(x, act):
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)
    s = 1.0 / (1.0 + torch.exp(-1.702 * x))
    return s * (1.0 + 1.702 * x * (1.0 - s))


def _run_plain(st):
    case = st["case"]
    if case["kind"].startswith("attn"):
        return _plain_attn(st)
    if case["kind"] == "embed":
        return _plain_embed(st)
    kept = _plain_kept(st["x"])
    if case["kind"] == "linear8":
        return {"dw": torch.matmul(st["dy"].float().t(), _plain_act(kept, case["act"])).to(DTYPES[case["grad"]])}
    x, dy = st["x"], st["dy"]
    return {"out": _plain_act(x.float(), case["act"]).to(x.dtype),
            "dx": (dy.float() * _plain_act_slope(kept, case["act"])).to(x.dtype)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ the floor

def _pairs(case):
    """(query, key) pairs that see each other, over the case's sequences, for one head."""
    lens = _lengths(case).astype(np.float64)
    if case["kind"] == "attn_token":
        return float(lens.sum())
    return float((lens * (lens + 1) / 2).sum() if case["causal"] else (lens * lens).sum())


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind.startswith("attn"):
        tk = float(_lengths(case).sum())
        tq = float(case["n"]) if kind == "attn_token" else tk
        rows_q, rows_k = tq * case["heads"] * case["hd"] * es, tk * case["kv"] * case["hd"] * es
        per = _pairs(case) * case["heads"] * case["hd"]
        if kind == "attn_train":  # q, k, v, dout in; out, dq, dk, dv out; two products forward, five backward
            return {"bytes": 4 * rows_q + 4 * rows_k, "flops": 14 * per}
        lse = tq * case["heads"] * 4 if kind == "attn_fwd" else 0
        return {"bytes": 2 * rows_q + 2 * rows_k + lse, "flops": 4 * per}
    if kind == "embed":
        n, d, ids = case["n"], case["d"], 4 if case["ids"] == "i32" else 8
        rows = min(n, case["vocab"])
        return {"bytes": n * ids + rows * d * es + 2 * n * d * es + case["vocab"] * d * 4, "flops": 2.0 * n * d}
    n, d = case["n"], case["d"]
    if kind == "linear8":  # x and dy in, dw out; the checkpoint written and read
        m = case["m"]
        g = 4 if case["grad"] == "f32" else 2
        return {"bytes": n * d * (es + 2 + 2.0 / GROUP) + n * m * es + m * d * g, "flops": 2.0 * n * d * m}
    # x, dy in; out, dx out; the checkpoint written and read
    return {"bytes": n * d * (4 * es + 2 + 2.0 / GROUP), "flops": 30.0 * n * d}


# ------------------------------------------------- the definitions in 64 bits

def _exact_attn(st):
    case = st["case"]
    q, k, v = (st[x].double() for x in ("q", "k", "v"))
    group = case["heads"] // case["kv"]
    train = case["kind"] == "attn_train"
    outs, lses, dqs, dks, dvs = [], [], [], [], []
    cq, ck = st["cu_q"].tolist(), st["cu_k"].tolist()
    for z in range(case["n"]):
        a, b = q[cq[z]:cq[z + 1]].transpose(0, 1), k[ck[z]:ck[z + 1]].repeat_interleave(group, 1).transpose(0, 1)
        c = v[ck[z]:ck[z + 1]].repeat_interleave(group, 1).transpose(0, 1)
        m, n = a.shape[1], b.shape[1]
        if n == 0:
            outs.append(torch.zeros((m, case["heads"], case["hd"]), dtype=torch.float64, device=q.device))
            lses.append(torch.full((case["heads"], m), -math.inf, dtype=torch.float64, device=q.device))
            if train:
                dqs.append(outs[-1])
                dks.append(k[:0])
                dvs.append(v[:0])
            continue
        if train:
            a, b, c = (t.contiguous().requires_grad_() for t in (a, b, c))
        s = torch.matmul(a, b.transpose(1, 2)) / math.sqrt(case["hd"])
        if case["causal"]:
            s = s + torch.triu(torch.full((m, n), -math.inf, dtype=torch.float64, device=q.device), n - m + 1)
        o = torch.matmul(torch.softmax(s, -1), c)
        if case["kind"] == "attn_fwd":
            lses.append(torch.logsumexp(s, -1))
        if train:
            da, db, dc = torch.autograd.grad(o, (a, b, c), st["dout"][cq[z]:cq[z + 1]].double().transpose(0, 1))
            dqs.append(da.transpose(0, 1))
            dks.append(db.view(case["kv"], group, n, -1).sum(1).transpose(0, 1))
            dvs.append(dc.view(case["kv"], group, n, -1).sum(1).transpose(0, 1))
        outs.append(o.detach().transpose(0, 1))
    res = {"out": torch.cat(outs)}
    if case["kind"] == "attn_fwd":
        res["lse"] = torch.cat(lses, 1)
    if train:
        res["dq"], res["dk"], res["dv"] = torch.cat(dqs), torch.cat(dks), torch.cat(dvs)
    return res


def _exact_kept(x):
    """x as its 8-bit checkpoint stands for it, group by group."""
    y = x.double()
    parts = []
    for g in y.split(GROUP, 1):
        top = g.abs().max(1, keepdim=True).values
        e = torch.where(top > 0, torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 6, -126.0)
        e = torch.where(torch.exp2(e) * 127.5 <= top, e + 1, e)  # (a tie at 127.5 rounds to 128)
        unit = torch.exp2(e.clamp(min=-126))
        parts.append(torch.round(g / unit) * unit)
    return torch.cat(parts, 1)


def _exact_act(x, act):
    if act == "gelu":
        return x * torch.special.ndtr(x)
    return x * torch.sigmoid(1.702 * x) if act == "quick_gelu" else x


def exact(case, seed):
    if case["kind"].startswith("attn") and _pairs(case) * case["heads"] * case["hd"] > 2e11:
        return None
    st = prepare(case, seed)
    if case["kind"].startswith("attn"):
        return _exact_attn(st)
    if case["kind"] == "embed":
        ids = st["tokens"].long()
        dtable = torch.zeros((case["vocab"], case["d"]), dtype=torch.float64, device=ids.device)
        dtable.index_add_(0, ids, st["dout"].double(), alpha=case["scale"])
        return {"out": st["table"].double()[ids] * case["scale"], "dtable": dtable}
    kept = _exact_kept(st["x"])
    if case["kind"] == "linear8":
        return {"dw": torch.matmul(st["dy"].double().t(), _exact_act(kept, case["act"]))}
    kept.requires_grad_()
    (dx,) = torch.autograd.grad(_exact_act(kept, case["act"]), kept, st["dy"].double())
    return {"out": _exact_act(st["x"].double(), case["act"]), "dx": dx}
