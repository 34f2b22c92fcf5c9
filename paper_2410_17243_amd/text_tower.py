"""A text tower on the library's operators: the encoder beside the tiled loss.

    python -m paper_2410_17243_amd.text_tower [--captions N] [--chunk C] [--steps K] [--rotary] [--dropout P]
        [--gates G] [--post-norms] [--products fp8]

Captions of different lengths are packed without padding.  A token embedding
and a position embedding (embed: their gradients by sorted tokens), causal
attention over the packed captions (packed_attn_qkv), the layers' inputs and
the activations kept in 8 bits (linear8, mlp8), and the feature of each
caption's last token.  It is a torch module whose input is a PackedCaptions, so
gradcache_step drives it, a chunk of captions at a time, with the tiled loss on
top; extend() takes one more token of every caption over a cache of keys and
values.

By choice: rotary positions instead of learned ones (rotary), dropout of what the
blocks add, gates and norms of it, with the residual sum and the next norm in one pass
(add_norm), and products of 8-bit floats (linear_fp8; the activation between them is
torch's and keeps 16 bits).  Dropout's masks are functions of the tower's seed, the layer,
and the token's place in the whole batch, so both passes of the gradient cache have the
same ones, however the batch is cut.

The command trains a small random-initialised tower against fixed random image
embeddings for a few steps and prints the loss and what a chunk keeps for its backward
pass.
"""

from __future__ import annotations

import argparse

import numpy as np
import torch

from . import (add_norm, embed, fp8_pack, linear8, linear_fp8, mlp8, packed_attn_fwd, packed_attn_qkv, rotary,
               rotary_freqs)


class PackedCaptions:
    """n captions as one vector of token ids.  cu [n + 1] int32: where each begins;
    lens: their lengths on the host (at least one token each).  first: the number of
    their first token, where they are a range of more captions."""

    def __init__(self, tokens, lens, first=0):
        self.tokens, self.lens, self.first = tokens, np.asarray(lens, dtype=np.int64), first
        if self.lens.ndim != 1 or (self.lens < 1).any() or int(self.lens.sum()) != tokens.numel():
            raise ValueError("lens must be the captions' lengths, each at least 1, of all tokens together")
        self.off = np.concatenate([[0], np.cumsum(self.lens)])
        self.max_len = int(self.lens.max()) if len(self.lens) else 0
        self.cu = torch.from_numpy(self.off.astype(np.int32)).to(tokens.device)

    @property
    def shape(self):
        return (len(self.lens),)

    def __getitem__(self, s):
        if not isinstance(s, slice):
            raise TypeError("captions are taken by ranges")
        a, b, step = s.indices(len(self.lens))
        if step != 1:
            raise ValueError("captions are taken by ranges without a step")
        b = max(a, b)
        return PackedCaptions(self.tokens[int(self.off[a]):int(self.off[b])], self.lens[a:b], self.first + int(self.off[a]))

    def positions(self):
        """Each token's place in its caption."""
        first = torch.repeat_interleave(self.cu[:-1], self.cu[1:] - self.cu[:-1], output_size=self.tokens.numel())
        return torch.arange(self.tokens.numel(), device=self.tokens.device, dtype=torch.int32) - first


class _Block(torch.nn.Module):
    def __init__(self, width, heads, kv_heads, act, dtype, gates=None, post_norms=False, products="16bit"):
        super().__init__()
        hd = width // heads
        self.heads, self.kv_heads, self.hd, self.act = heads, kv_heads, hd, act
        new = lambda *s: torch.nn.Parameter((torch.randn(s) / s[-1] ** 0.5).to(dtype))  # noqa: E731
        zero = lambda n: torch.nn.Parameter(torch.zeros(n, dtype=dtype))  # noqa: E731
        self.qkv_w, self.qkv_b = new((heads + 2 * kv_heads) * hd, width), zero((heads + 2 * kv_heads) * hd)
        self.out_w, self.out_b = new(width, width), zero(width)
        self.w1, self.b1, self.w2, self.b2 = new(4 * width, width), zero(4 * width), new(width, 4 * width), zero(width)
        self.n1, self.n2 = torch.nn.LayerNorm(width, dtype=dtype), torch.nn.LayerNorm(width, dtype=dtype)
        self.products = products
        gate = lambda: None if gates is None else torch.nn.Parameter(torch.full((width,), gates, dtype=dtype))  # noqa: E731
        self.g1, self.g2 = gate(), gate()
        self.p1, self.p2 = (torch.nn.LayerNorm(width, dtype=dtype) if post_norms else None for _ in range(2))

    def qkv(self, x):
        return self.heads_of(linear8(self.n1(x), self.qkv_w, self.qkv_b))

    def heads_of(self, y):
        return y.view(-1, self.heads + 2 * self.kv_heads, self.hd)

    def packed(self, dtype):
        """The weights, as layers of dtype take them, in 8-bit floats, for calls without gradients."""
        return {k: fp8_pack(getattr(self, k).detach().to(dtype)) for k in ("qkv_w", "out_w", "w1", "w2")}

    def layer(self, x, w, b, packed=None):
        if self.products == "16bit":
            return linear8(x, getattr(self, w), getattr(self, b))
        return linear_fp8(x, packed[w] if packed else getattr(self, w), getattr(self, b))

    def mlp(self, z, packed=None):
        if self.products == "16bit":
            return mlp8(z, self.w1, self.b1, self.w2, self.b2, self.act)
        t = self.layer(z, "w1", "b1", packed)
        t = torch.nn.functional.gelu(t) if self.act == "gelu" else t * torch.sigmoid(1.702 * t)
        return self.layer(t, "w2", "b2", packed)

    def rest(self, x, a):
        x = x + linear8(a.reshape(x.shape), self.out_w, self.out_b)
        return x + mlp8(self.n2(x), self.w1, self.b1, self.w2, self.b2, self.act)


class TextTower(torch.nn.Module):
    """Captions (PackedCaptions) -> unit rows [n, out_dim]."""

    def __init__(self, vocab, width, layers, heads, out_dim, max_len, kv_heads=None, act="quick_gelu",
                 dtype=torch.bfloat16, rotary=False, dropout=0.0, gates=None, post_norms=False, products="16bit"):
        """gates: the first value of what each feature of a block's output is multiplied
        with; post_norms: a norm of that output.  seed (an attribute; an int, or an int64
        tensor of one element) is dropout's, to be changed from step to step."""
        super().__init__()
        if products not in ("16bit", "fp8"):
            raise ValueError(f'products must be "16bit" or "fp8", got {products!r}')
        if act not in ("gelu", "quick_gelu"):
            raise ValueError(f'act must be "gelu" or "quick_gelu", got {act!r}')
        if not 0.0 <= dropout < 1.0:
            raise ValueError(f"dropout must be from 0 to below 1, got {dropout}")
        if width % heads or (width // heads) % 8 or width // heads > 128:
            raise ValueError(f"width {width} must be heads times a multiple of 8 up to 128, got {heads} heads")
        self.max_len = max_len
        self.table = torch.nn.Parameter((0.02 * torch.randn(vocab, width)).to(dtype))
        self.places = None if rotary else torch.nn.Parameter((0.01 * torch.randn(max_len, width)).to(dtype))
        self.register_buffer("freqs", rotary_freqs(width // heads // 2, device="cpu") if rotary else None, persistent=False)
        self.dropout, self.seed = dropout, 0
        self.fused = dropout > 0 or gates is not None or post_norms or products == "fp8"
        self.blocks = torch.nn.ModuleList(_Block(width, heads, kv_heads or heads, act, dtype, gates, post_norms, products)
                                          for _ in range(layers))
        self.norm = torch.nn.LayerNorm(width, dtype=dtype)
        self.proj = torch.nn.Parameter((torch.randn(out_dim, width) / width ** 0.5).to(dtype))

    def _apply(self, fn, *args, **kw):
        """.to(), .half() and their like: the frequencies move with the parameters and stay
        fp32, the same bits (8 bits of a frequency are 0.007 rad at position 39)."""
        freqs = self.freqs
        super()._apply(fn, *args, **kw)
        if freqs is not None:
            dev = self.freqs.device
            self.freqs = rotary_freqs(freqs.numel(), device=dev) if freqs.is_meta else freqs.to(dev)
        return self

    @property
    def dtype(self):
        return self.table.dtype

    def _block_dtype(self):
        """What the blocks' layers compute in."""
        return torch.get_autocast_dtype("cuda") if torch.is_autocast_enabled("cuda") else self.dtype

    def _features(self, x):
        return self._project(self.norm(x))

    def _project(self, z):
        return torch.nn.functional.normalize(torch.nn.functional.linear(z, self.proj).float(), dim=-1)

    def forward(self, captions: PackedCaptions):
        if captions.max_len > self.max_len:
            raise ValueError(f"captions of up to {captions.max_len} tokens, the tower takes {self.max_len}")
        x, pos = self._rows(captions.tokens, captions.positions())

        def attend(b, i, qkv):
            return packed_attn_qkv(self._turned(b, qkv, pos), b.heads, b.kv_heads, captions.cu, captions.max_len)

        last = captions.cu[1:].long() - 1
        if self.fused:
            return self._project(self._through(x, attend, captions.first)[last])
        for i, b in enumerate(self.blocks):
            x = b.rest(x, attend(b, i, b.qkv(x)))
        return self._features(x[last])

    def _rows(self, tokens, pos):
        x = embed(tokens, self.table)
        return x if self.places is None else x + embed(pos, self.places), pos

    def _turned(self, b, qkv, pos):
        return qkv if self.freqs is None else rotary(qkv, pos, self.freqs, turned=b.heads + b.kv_heads)

    def _through(self, x, attend, first=0, packed=None):
        """The blocks with add_norm between them: rows after the last norm."""
        drop = {"p": self.dropout if self.training and packed is None else 0.0, "seed": self.seed, "row0": first}
        blocks = list(self.blocks)
        nexts = [b.n1 for b in blocks[1:]] + [self.norm]

        def add(x, y, post, gate, pre, site):
            w = (None, None) if post is None else (post.weight, post.bias)
            # (under autocast the blocks' outputs have 16 bits, the residual rows those of the table)
            return add_norm(x, y.to(x.dtype), gate, *w, pre.weight, pre.bias, eps=pre.eps, site=site, **drop)

        z = add_norm(x, pre_w=blocks[0].n1.weight, pre_b=blocks[0].n1.bias, eps=blocks[0].n1.eps)[1] if blocks else None
        for i, (b, after) in enumerate(zip(blocks, nexts)):
            p = packed[i] if packed else None
            a = attend(b, i, b.heads_of(b.layer(z, "qkv_w", "qkv_b", p)))
            x, z = add(x, b.layer(a.reshape(x.shape), "out_w", "out_b", p), b.p1, b.g1, b.n2, 2 * i)
            x, z = add(x, b.mlp(z, p), b.p2, b.g2, after, 2 * i + 1)
        return self.norm(x) if z is None else z

    def new_cache(self, n: int):
        """Room for the keys and values of n captions, empty; with products of 8-bit floats
        also the weights packed as they are now.  It is for calls of extend under the
        autocast that it was made under, or none."""
        dev, dtype = self.table.device, self._block_dtype()
        cu = torch.arange(n + 1, dtype=torch.int32, device=dev)
        kv = [torch.zeros((2, n * self.max_len, b.kv_heads, b.hd), dtype=dtype, device=dev) for b in self.blocks]
        packed = [b.packed(dtype) if b.products == "fp8" else {} for b in self.blocks]
        return {"kv": kv, "cu_q": cu, "cu_k": cu * self.max_len, "len": torch.zeros(n, dtype=torch.int32, device=dev),
                "taken": 0, "packed": packed, "dtype": dtype}

    @torch.no_grad()
    def extend(self, tokens, cache):
        """One more token of every caption (tokens [n]): its feature rows, as forward
        gives them for the captions so far; keys and values go to the cache, which
        has room for max_len tokens of each."""
        if cache["taken"] == self.max_len or tokens.numel() != cache["len"].numel():
            raise ValueError(f"a token for each of {cache['len'].numel()} captions, {self.max_len} times at most")
        if cache["dtype"] != self._block_dtype():
            raise ValueError(f"the cache is of {cache['dtype']}, the blocks compute in {self._block_dtype()}: make it where it is used")
        cache["taken"] += 1
        at = cache["cu_k"][:-1].long() + cache["len"].long()
        x, pos = self._rows(tokens, cache["len"].clone())
        cache["len"] += 1

        def attend(b, i, qkv):
            kv = cache["kv"][i]
            qkv = self._turned(b, qkv, pos)
            q, k, v = qkv[:, :b.heads], qkv[:, b.heads:b.heads + b.kv_heads], qkv[:, b.heads + b.kv_heads:]
            kv[0][at], kv[1][at] = k, v
            return packed_attn_fwd(q, kv[0], kv[1], cache["cu_q"], 1, cache["cu_k"], self.max_len, need_lse=False,
                                   len_k=cache["len"])[0]

        if self.fused:
            return self._project(self._through(x, attend, packed=cache["packed"]))
        for i, b in enumerate(self.blocks):
            x = b.rest(x, attend(b, i, b.qkv(x)))
        return self._features(x)


def synthetic_captions(n, vocab, max_len, seed=0, device="cuda"):
    """n captions of lognormal lengths around 16, Zipf-like tokens between the
    first id (opening) and the last (closing)."""
    rs = np.random.RandomState(seed)
    lens = np.clip(np.rint(np.exp(rs.normal(np.log(16.0), 0.5, n))), 3, max_len).astype(np.int64)
    t = np.minimum(np.exp(rs.rand(int(lens.sum())) * np.log(vocab)).astype(np.int64), vocab - 2)
    end = np.cumsum(lens)
    t[end - lens], t[end - 1] = 0, vocab - 1
    return PackedCaptions(torch.from_numpy(t).to(device), lens)


def main():
    from .gradcache import gradcache_step

    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--captions", type=int, default=4096)
    ap.add_argument("--chunk", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--rotary", action="store_true")
    ap.add_argument("--dropout", type=float, default=0.0)
    ap.add_argument("--gates", type=float, default=None)
    ap.add_argument("--post-norms", action="store_true")
    ap.add_argument("--products", choices=["16bit", "fp8"], default="16bit")
    a = ap.parse_args()
    torch.manual_seed(0)
    tower = TextTower(49152, a.width, a.layers, a.width // 64, 512, 77, rotary=a.rotary, dropout=a.dropout, gates=a.gates,
                      post_norms=a.post_norms, products=a.products).cuda()
    captions = synthetic_captions(a.captions, 49152, 77)
    images = torch.nn.functional.normalize(torch.randn(a.captions, 512, device="cuda"), dim=-1)
    image_side = torch.nn.Linear(512, 512, device="cuda")
    scale = torch.tensor(14.29, device="cuda")
    opt = torch.optim.Adam([*tower.parameters(), *image_side.parameters()], lr=3e-4, eps=1e-6)
    before = torch.cuda.memory_allocated()
    kept = tower(captions[:a.chunk])
    print(f"{a.captions} captions, {captions.tokens.numel()} tokens; a chunk of {a.chunk} keeps "
          f"{(torch.cuda.memory_allocated() - before) / 2 ** 20:.1f} MiB for its backward pass")
    del kept
    for i in range(a.steps):
        opt.zero_grad(set_to_none=True)
        tower.seed = i
        loss, _ = gradcache_step(image_side, tower, images, captions, scale, a.chunk)
        opt.step()
        print(f"step {i}: loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
