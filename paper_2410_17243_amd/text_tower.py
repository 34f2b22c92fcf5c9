"""A text tower on the library's operators: the encoder beside the tiled loss.

    python -m paper_2410_17243_amd.text_tower [--captions N] [--chunk C] [--steps K]

Captions of different lengths are packed without padding.  A token embedding
and a position embedding (embed: their gradients by sorted tokens), causal
attention over the packed captions (packed_attn_qkv), the layers' inputs and
the activations kept in 8 bits (linear8, mlp8), and the feature of each
caption's last token.  It is a torch module whose input is a PackedCaptions, so
gradcache_step drives it, a chunk of captions at a time, with the tiled loss on
top; extend() takes one more token of every caption over a cache of keys and
values.  The command trains a small random-initialised tower against fixed
random image embeddings for a few steps and prints the loss and what a chunk
keeps for its backward pass.
"""

from __future__ import annotations

import argparse

import numpy as np
import torch

from . import embed, linear8, mlp8, packed_attn_fwd, packed_attn_qkv


class PackedCaptions:
    """n captions as one vector of token ids.  cu [n + 1] int32: where each begins;
    lens: their lengths on the host (at least one token each)."""

    def __init__(self, tokens, lens):
        self.tokens, self.lens = tokens, np.asarray(lens, dtype=np.int64)
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
        return PackedCaptions(self.tokens[int(self.off[a]):int(self.off[b])], self.lens[a:b])

    def positions(self):
        """Each token's place in its caption."""
        first = torch.repeat_interleave(self.cu[:-1], self.cu[1:] - self.cu[:-1], output_size=self.tokens.numel())
        return torch.arange(self.tokens.numel(), device=self.tokens.device, dtype=torch.int32) - first


class _Block(torch.nn.Module):
    def __init__(self, width, heads, kv_heads, act, dtype):
        super().__init__()
        hd = width // heads
        self.heads, self.kv_heads, self.hd, self.act = heads, kv_heads, hd, act
        new = lambda *s: torch.nn.Parameter((torch.randn(s) / s[-1] ** 0.5).to(dtype))  # noqa: E731
        zero = lambda n: torch.nn.Parameter(torch.zeros(n, dtype=dtype))  # noqa: E731
        self.qkv_w, self.qkv_b = new((heads + 2 * kv_heads) * hd, width), zero((heads + 2 * kv_heads) * hd)
        self.out_w, self.out_b = new(width, width), zero(width)
        self.w1, self.b1, self.w2, self.b2 = new(4 * width, width), zero(4 * width), new(width, 4 * width), zero(width)
        self.n1, self.n2 = torch.nn.LayerNorm(width, dtype=dtype), torch.nn.LayerNorm(width, dtype=dtype)

    def qkv(self, x):
        return linear8(self.n1(x), self.qkv_w, self.qkv_b).view(-1, self.heads + 2 * self.kv_heads, self.hd)

    def rest(self, x, a):
        x = x + linear8(a.reshape(x.shape), self.out_w, self.out_b)
        return x + mlp8(self.n2(x), self.w1, self.b1, self.w2, self.b2, self.act)


class TextTower(torch.nn.Module):
    """Captions (PackedCaptions) -> unit rows [n, out_dim]."""

    def __init__(self, vocab, width, layers, heads, out_dim, max_len, kv_heads=None, act="quick_gelu",
                 dtype=torch.bfloat16):
        super().__init__()
        if width % heads or (width // heads) % 8 or width // heads > 128:
            raise ValueError(f"width {width} must be heads times a multiple of 8 up to 128, got {heads} heads")
        self.max_len, self.dtype = max_len, dtype
        self.table = torch.nn.Parameter((0.02 * torch.randn(vocab, width)).to(dtype))
        self.places = torch.nn.Parameter((0.01 * torch.randn(max_len, width)).to(dtype))
        self.blocks = torch.nn.ModuleList(_Block(width, heads, kv_heads or heads, act, dtype) for _ in range(layers))
        self.norm = torch.nn.LayerNorm(width, dtype=dtype)
        self.proj = torch.nn.Parameter((torch.randn(out_dim, width) / width ** 0.5).to(dtype))

    def _features(self, x):
        y = torch.nn.functional.linear(self.norm(x), self.proj).float()
        return torch.nn.functional.normalize(y, dim=-1)

    def forward(self, captions: PackedCaptions):
        if captions.max_len > self.max_len:
            raise ValueError(f"captions of up to {captions.max_len} tokens, the tower takes {self.max_len}")
        x = embed(captions.tokens, self.table) + embed(captions.positions(), self.places)
        for b in self.blocks:
            x = b.rest(x, packed_attn_qkv(b.qkv(x), b.heads, b.kv_heads, captions.cu, captions.max_len))
        return self._features(x[captions.cu[1:].long() - 1])

    def new_cache(self, n: int):
        """Room for the keys and values of n captions, empty."""
        dev = self.table.device
        cu = torch.arange(n + 1, dtype=torch.int32, device=dev)
        kv = [torch.zeros((2, n * self.max_len, b.kv_heads, b.hd), dtype=self.dtype, device=dev) for b in self.blocks]
        return {"kv": kv, "cu_q": cu, "cu_k": cu * self.max_len, "len": torch.zeros(n, dtype=torch.int32, device=dev),
                "taken": 0}

    @torch.no_grad()
    def extend(self, tokens, cache):
        """One more token of every caption (tokens [n]): its feature rows, as forward
        gives them for the captions so far; keys and values go to the cache, which
        has room for max_len tokens of each."""
        if cache["taken"] == self.max_len or tokens.numel() != cache["len"].numel():
            raise ValueError(f"a token for each of {cache['len'].numel()} captions, {self.max_len} times at most")
        cache["taken"] += 1
        at = cache["cu_k"][:-1].long() + cache["len"].long()
        x = embed(tokens, self.table) + embed(cache["len"], self.places)
        cache["len"] += 1
        for b, kv in zip(self.blocks, cache["kv"]):
            qkv = b.qkv(x)
            q, k, v = qkv[:, :b.heads], qkv[:, b.heads:b.heads + b.kv_heads], qkv[:, b.heads + b.kv_heads:]
            kv[0][at], kv[1][at] = k, v
            a, _ = packed_attn_fwd(q, kv[0], kv[1], cache["cu_q"], 1, cache["cu_k"], self.max_len, need_lse=False,
                                   len_k=cache["len"])
            x = b.rest(x, a)
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
    a = ap.parse_args()
    torch.manual_seed(0)
    tower = TextTower(49152, a.width, a.layers, a.width // 64, 512, 77).cuda()
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
        loss, _ = gradcache_step(image_side, tower, images, captions, scale, a.chunk)
        opt.step()
        print(f"step {i}: loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
