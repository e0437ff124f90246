"""A streamed latent predictor in front of the decoder chain: the token operators as a world model would run them.

A small transformer predicts a latent frame of H x W tokens from the frames before it, one frame a call, and the decoder
chain (``chain.ResidentDecoderChain``) turns each predicted frame into four output frames.  As in the chain, the weights
are random and there is no claim about what it predicts; it shows the operators together:

    per block   h = pre-norm of the residual, scaled and shifted for the frame    gated_norm
                q, k, v = h Wqkv          (one library product)
                keys and values into the paged cache, q and k rotated by (frame, row, column)      PagedCache.append
                attention over the frames so far, causal in frames, a window of frames             PagedCache.attend
                residual += gate * norm(attention Wo); h = pre-norm ...                            gated_norm
                residual += gate * norm(silu(h W1) W2)                                             (with the next block's)

The cache is paged: pages of frames that have left the window go back to the pool, so a stream of any length runs in a
fixed amount of memory, as the chain does with its frame rings.  Its rotation tables are of a fixed length, too: along the
frames, pairs turn by whole numbers of turns in as many frames as a table has rows, so that a frame's row is its number
modulo the rows and the angle between two frames is that of their distance wherever the stream stands.

``DecayPredictor`` is the same with a memory of fixed size, one state for each head that old frames fade from, in place of the
cache, and with every product in the library:

    per block   h = pre-norm of the residual, scaled and shifted for the frame                 gated_norm
                q, k, v = h Wqkv, log decays from h Wg                                         linear
                the frame's tokens into the states, read in their order                        DecayMemory.attend
                residual += (norm of each head) Wo                                             group_norm, linear
                h = pre-norm ...; residual += (silu(h W1) * (h W2)) W3                         gated_norm, linear (gated), linear

    python -m paper_2609_31938_b200.predictor [frames] [cache | decay]
"""
from __future__ import annotations

import math

import torch

from . import tokens as tk


class LatentPredictor:
    def __init__(self, channels=192, heads=6, kv_heads=2, head_dim=64, blocks=2, height=44, width=80, window_frames=4,
                 page_tokens=64, seed=0, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s, a=1.0: torch.randn(s, generator=g, device="cuda") * a  # noqa: E731
        self.c, self.hq, self.hk, self.d = channels, heads, kv_heads, head_dim
        self.h, self.w, self.n = height, width, height * width
        self.window, self.page, self.dtype = window_frames, page_tokens, dtype
        qkv, inner = (heads + 2 * kv_heads) * head_dim, 4 * channels
        self.blocks = [dict(qkv=rnd(channels, qkv, a=channels ** -0.5).to(dtype), out=rnd(heads * head_dim, channels, a=(heads * head_dim) ** -0.5).to(dtype),
                            up=rnd(channels, inner, a=channels ** -0.5).to(dtype), down=rnd(inner, channels, a=inner ** -0.5).to(dtype),
                            w=[1 + rnd(channels, a=0.1) for _ in range(4)]) for _ in range(blocks)]
        # gate, scale and shift of each half block from the frame's conditioning
        self.modulation = rnd(channels, blocks * 6 * channels, a=0.3 * channels ** -0.5)
        pairs = head_dim // 2
        sections = (pairs - 2 * (pairs * 3 // 8), pairs * 3 // 8, pairs * 3 // 8)
        rows = max(256, height, width, 8 * (window_frames + 1))
        speed = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)         # radians a step
        turns = (speed[:sections[0]] * rows / (2 * math.pi)).round().clamp_min(1)      # along the frames: in `rows` of them
        steps = torch.arange(rows, dtype=torch.float64)[:, None]
        angle = steps * speed
        angle[:, :sections[0]] = steps * turns % rows * (2 * math.pi / rows)
        self.rotary = tk.Rotary(angle.cos().float().cuda(), angle.sin().float().cuda(), sections)
        self.rows = rows
        # pages of window_frames + 1 frames (and one that a frame's border cuts), one table for all blocks
        self.table_pages = -(-(window_frames + 1) * self.n // page_tokens) + 2
        self.caches = [tk.PagedCache.empty(self.table_pages, kv_heads, head_dim, page_tokens) for _ in range(blocks)]
        self._reported = [0] * blocks                  # by caches that the pool outgrew
        self.reset()

    def reset(self):
        """Forget the stream (the next frame is the first)."""
        self.frame, self.origin = 0, 0                 # frames seen; first frame that the table still covers
        self.free = list(range(self.table_pages))
        self.held = []                                 # pages of the tokens from frame `origin` on

    def _batch(self):
        """Table and lengths for the next frame.  Frames that left the window go; positions in the cache count from the oldest
        frame that is left, which starts a page only if a whole number of pages was given back."""
        n, page = self.n, self.page
        step = page // math.gcd(n, page)               # frames whose tokens fill whole pages
        while self.frame - self.origin >= self.window + step:
            drop = step * n // page
            self.free += self.held[:drop]
            self.held = self.held[drop:]
            self.origin += step
        total = (self.frame - self.origin + 1) * n
        while len(self.held) * page < total:
            if not self.free:                          # a frame that is no whole number of pages keeps its neighbours longer
                grow = self.table_pages
                for i, c in enumerate(self.caches):
                    self._reported[i] |= c.status()
                    self.caches[i] = tk.PagedCache(torch.cat([c.codes, torch.empty_like(c.codes[:grow])]), torch.cat([c.scales, torch.zeros_like(c.scales[:grow])]))
                self.free = list(range(self.caches[0].pages - grow, self.caches[0].pages))
            self.held.append(self.free.pop(0))
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        return tk.TokenBatch(ints([0, n]), ints([total]), ints([self.held]), max_new=n)

    def status(self):
        """TOKENS_* bits that the kernels have reported for each block's cache, cleared by reading (waits for the device)."""
        bits = [c.status() | r for c, r in zip(self.caches, self._reported)]
        self._reported = [0] * len(bits)
        return bits

    def step(self, x, condition):
        """One frame: x [H * W, channels] (noise, or what a caller has of the frame) and condition [channels] ->
        the predicted latent frame [H * W, channels]."""
        n, c = self.n, self.c
        batch = self._batch()
        t = torch.arange(n, device="cuda", dtype=torch.int32)
        pos = torch.stack([torch.full_like(t, self.frame % self.rows), t // self.w, t % self.w], 1)
        mod = (condition.float() @ self.modulation).view(len(self.blocks), 2, 3, 1, c)
        w0 = self.blocks[0]["w"]
        r, h = tk.gated_norm(x.float(), None, pre_weight=w0[0], scale=mod[0, 0, 1], shift=mod[0, 0, 2], act_dtype=self.dtype)
        for i, (b, cache) in enumerate(zip(self.blocks, self.caches)):
            qkv = (h @ b["qkv"]).view(n, self.hq + 2 * self.hk, self.d)
            q, k, v = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hk], qkv[:, self.hq + self.hk:]
            q = cache.append(k, v, batch, self.rotary, pos, q=q, q_out=q)
            a = cache.attend(q, batch, frame=n, window=self.window * n)
            # between attention and feed-forward, then between this block and the next
            r, h = tk.gated_norm(r, a.view(n, -1) @ b["out"], gate=mod[i, 0, 0], post_weight=b["w"][1], post_kind="rms",
                                 pre_weight=b["w"][2], scale=mod[i, 1, 1], shift=mod[i, 1, 2], out_r=r)
            y = torch.nn.functional.silu(h @ b["up"]) @ b["down"]
            last = i + 1 == len(self.blocks)
            nxt = None if last else self.blocks[i + 1]["w"][0]
            r, h = tk.gated_norm(r, y, gate=mod[i, 1, 0], post_weight=b["w"][3], post_kind="rms", pre_weight=nxt,
                                 scale=None if last else mod[i + 1, 0, 1], shift=None if last else mod[i + 1, 0, 2],
                                 out_r=r, want_h=not last)
        self.frame += 1
        return r

    def latent(self, r):
        """[H * W, channels] -> [1, channels, 1, H, W] in BF16, the decoder chain's input."""
        return r.view(1, 1, self.h, self.w, self.c).permute(0, 4, 1, 2, 3).to(torch.bfloat16).contiguous()


class DecayPredictor:
    def __init__(self, channels=192, heads=6, key_dim=64, value_dim=64, blocks=2, height=44, width=80, seed=0, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s, a=1.0: torch.randn(s, generator=g, device="cuda") * a  # noqa: E731
        self.c, self.heads, self.dk, self.dv = channels, heads, key_dim, value_dim
        self.h, self.w, self.n, self.dtype = height, width, height * width, dtype
        inner = 4 * channels
        self.blocks = [dict(qkv=rnd(heads * (2 * key_dim + value_dim), channels, a=channels ** -0.5).to(dtype),
                            decay=rnd(heads, channels, a=0.3 * channels ** -0.5).to(dtype),
                            # heads that remember from a part of a frame to several frames
                            rate=-torch.linspace(4.0, 11.0, heads, device="cuda").to(dtype),
                            head=(1 + rnd(heads * value_dim, a=0.1), rnd(heads * value_dim, a=0.1)),
                            out=rnd(channels, heads * value_dim, a=(heads * value_dim) ** -0.5).to(dtype),
                            up=rnd(2 * inner, channels, a=channels ** -0.5).to(dtype), down=rnd(channels, inner, a=inner ** -0.5).to(dtype),
                            w=[1 + rnd(channels, a=0.1) for _ in range(2)]) for _ in range(blocks)]
        self.modulation = rnd(channels, blocks * 4 * channels, a=0.3 * channels ** -0.5)     # scale and shift of each half block
        self.memories = [tk.DecayMemory.empty(1, heads, key_dim, value_dim) for _ in range(blocks)]
        self._fresh = torch.ones(1, dtype=torch.int32, device="cuda")
        self.batch = tk.StreamBatch(torch.tensor([0, self.n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"),
                                    self.n, fresh=self._fresh)
        self.reset()

    def reset(self):
        """Forget the stream (the next frame is the first)."""
        self._fresh.fill_(1)

    def status(self):
        """TOKENS_* bits that the kernels have reported, for each block's states and for the products, cleared by reading."""
        return [m.status() for m in self.memories] + [tk.status()]

    def step(self, x, condition):
        """One frame: x [H * W, channels] and condition [channels] -> the predicted latent frame [H * W, channels] (float32)."""
        n, c, hk, hv = self.n, self.c, self.heads * self.dk, self.heads * self.dv
        mod = (condition.float() @ self.modulation).view(len(self.blocks), 2, 2, 1, c)
        r = x.float().clone()
        for i, (b, memory) in enumerate(zip(self.blocks, self.memories)):
            _, h = tk.gated_norm(r, pre_weight=b["w"][0], scale=mod[i, 0, 0], shift=mod[i, 0, 1], act_dtype=self.dtype, want_r=False)
            qkv = tk.linear(h, b["qkv"])
            q, k, v = qkv[:, :hk].unflatten(1, (self.heads, self.dk)), qkv[:, hk:2 * hk].unflatten(1, (self.heads, self.dk)), qkv[:, 2 * hk:].unflatten(1, (self.heads, self.dv))
            log_decay = -torch.nn.functional.softplus(tk.linear(h, b["decay"], b["rate"], out_dtype=torch.float32))
            o = memory.attend(q, k, v, log_decay, self.batch)
            o = tk.group_norm(o.view(n, 1, hv), self.heads, *b["head"])
            r = tk.linear(o.view(n, hv), b["out"], residual=r, out=r)
            _, h = tk.gated_norm(r, pre_weight=b["w"][1], scale=mod[i, 1, 0], shift=mod[i, 1, 1], act_dtype=self.dtype, want_r=False)
            u = tk.linear(h, b["up"], activation="silu", gated=True)
            r = tk.linear(u, b["down"], residual=r, out=r)
        self._fresh.zero_()
        return r

    latent = LatentPredictor.latent


def main(frames=6, memory="cache"):
    from .chain import LAYERS, NormedDecoderChain, ResidentDecoderChain
    g = torch.Generator(device="cuda").manual_seed(1)
    ca, cb, cc = 192, 96, 96
    shapes = {"A1": (ca, ca, 3), "A2": (ca, ca, 3), "PA": (cb, ca, 1), "B1": (cb, cb, 3), "B2": (cb, cb, 3), "PB": (cc, cb, 1),
              "C1": (cc, cc, 3), "C2": (cc, cc, 3)}
    w = {k: (torch.randn((co, ci, n, n, n), generator=g, device="cuda") * (ci * n ** 3) ** -0.5).bfloat16() for k, (co, ci, n) in shapes.items()}
    b = {k: torch.zeros(w[k].shape[0], device="cuda").bfloat16() for k in LAYERS}
    if memory == "decay":
        norms = {k: (torch.ones(shapes[k][1], device="cuda"), torch.zeros(shapes[k][1], device="cuda")) for k in LAYERS if k[0] != "P"}
        chain, model = NormedDecoderChain(w, b, norms), DecayPredictor(channels=ca)
    else:
        chain, model = ResidentDecoderChain(w, b), LatentPredictor(channels=ca)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for f in range(frames):
        noise, condition = torch.randn(model.n, ca, generator=g, device="cuda"), torch.randn(ca, generator=g, device="cuda")
        start.record()
        z = model.latent(model.step(noise, condition))
        out = chain.step(z)
        end.record()
        end.synchronize()
        print(f"frame {f}: {tuple(z.shape)} -> {tuple(out.shape)}, {start.elapsed_time(end):.2f} ms, rms {out.float().square().mean().sqrt().item():.3f}")
    bad = model.status()
    chain.close()
    if any(bad):
        raise SystemExit(f"reported by the cache kernels: {[hex(b) for b in bad]}")


if __name__ == "__main__":
    import sys
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 6, sys.argv[2] if len(sys.argv) > 2 else "cache")
