"""An attention context model on the wavefront schedule, its cache held in 4 bits.

The masked convolution of the context model is replaced by attention over every
latent decoded before: a step's latents are d-separated given the steps before
it (Sec. III-A, Eq. 4), so all of them attend to the same prefix of a cache that
is kept in step order.  A step
  - projects the hyperprior parameters psi of its latents to queries,
  - attends to the latents decoded so far (none in the first step),
  - predicts the means, codes (or decodes) the symbols: y_hat = symbol + mean,
  - projects y_hat and psi to keys and values, which join the cache in 4 bits.
Encoder and decoder run the same calls on the same values, so they see the same
quantised cache and their reconstructions agree bit for bit.  Weights are random:
the example shows the calls, not a trained model.

Options: `placed` norms queries and keys and rotates them by the latent's row and
column; `window` lets a latent see the last so many and the first `sinks` ones,
so that a step takes as long near the end of a grid as in its middle; `search`
tries several ways to code the next steps behind the latents that are coded.

    python examples/attention_context.py [H W M]
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_19082_amd import inputs, wf  # noqa: E402

HEAD = 64


class AttentionContext:
    def __init__(self, H, W, M, B=1, q_heads=None, heads=None, dtype=torch.bfloat16, page=64, seed=0,
                 placed=False, window=None, sinks=0, spare=0):
        if M % HEAD:
            raise ValueError(f"M must be a multiple of {HEAD}")
        self.H, self.W, self.M, self.B, self.dtype = H, W, M, B, dtype
        self.q_heads = q_heads or M // HEAD
        self.heads = heads or self.q_heads
        step, n_steps, _ = wf.schedule(H, W)
        flat = step.reshape(-1)
        order = np.argsort(flat, kind="stable")          # the cache's order: by step, then by row
        self.order = torch.from_numpy(order).cuda()
        self.bounds = np.searchsorted(flat[order], np.arange(n_steps + 1))
        rng = np.random.default_rng(seed)
        draw = lambda i, o: torch.from_numpy((rng.standard_normal((i, o)) / np.sqrt(i)).astype(np.float32)).cuda()  # noqa: E731
        self.wq = draw(2 * M, self.q_heads * HEAD)
        self.wk, self.wv = draw(3 * M, self.heads * HEAD), draw(3 * M, self.heads * HEAD)
        self.wo = draw(self.q_heads * HEAD, M)
        self.wp = draw(2 * M, M)
        per = -(-H * W // page)
        self.table = torch.arange(B * per, dtype=torch.int32, device="cuda").reshape(B, per)
        self.cache = wf.Cache(self.heads, HEAD, B * per + spare, page=page)
        self.spare = torch.arange(B * per, B * per + spare, dtype=torch.int32, device="cuda")    # pages that search may use
        self.window, self.sinks = window, sinks
        self.norm = wf.HeadNorm(HEAD, axes=2, base=100.0) if placed else None
        self.place = torch.from_numpy(np.stack([order // W, order % W], -1).astype(np.int32)).cuda()    # of each token: row, column

    def _heads(self, x, w, heads, a):
        """Rows x [B][n][..] of the latents from place a on as heads, normed and
        rotated where the model's are."""
        B, n, _ = x.shape
        h = (x @ w).to(self.dtype).view(B, n, heads, HEAD)
        if self.norm is None or w is self.wv:
            return h
        return self.norm.apply(h, self.place[a:a + n].expand(B, n, 2).contiguous(), out=h)

    def _write(self, y, p, table, a, first):
        x = torch.cat([y, p], -1)
        k, v = (self._heads(x, w, self.heads, a) for w in (self.wk, self.wv))
        self.cache.write(k, v, table, torch.full((len(x),), first, dtype=torch.int32, device="cuda"))

    def _run(self, psi, step_symbols, steps=None):
        """psi [B][H*W][2M] in cache order; step_symbols(a, b, mean) gives the
        symbols of places a to b.  Returns (symbols, y_hat) in cache order, of
        the first `steps` steps."""
        B = self.B
        symbols, y_hat = [], []
        for a, b in list(zip(self.bounds[:-1].tolist(), self.bounds[1:].tolist()))[:steps]:
            n, p = b - a, psi[:, a:b]
            q = self._heads(p, self.wq, self.q_heads, a)
            seen = torch.full((B, n), a, dtype=torch.int32, device="cuda")
            if self.window is None:
                ctx = self.cache.attend(q, self.table, seen, max_visible=a)
            else:
                ctx = self.cache.attend_window(q, self.table, seen, self.window, self.sinks, max_visible=a)
            mean = ctx.float().view(B, n, -1) @ self.wo + p @ self.wp
            s = step_symbols(a, b, mean)
            y = s + mean
            self._write(y, p, self.table, a, a)
            symbols.append(s)
            y_hat.append(y)
        return torch.cat(symbols, 1), torch.cat(y_hat, 1)

    def search(self, psi, y, step, ahead, offsets):
        """The squared errors of len(offsets) ways to code `ahead` steps of one image
        from `step` (at least 1) on, symbols = round(y - mean + offset), behind the
        steps before, which are coded as by encode.  The ways see the coded latents
        as a prefix that they share, and their own in spare pages."""
        if self.B != 1 or self.window is not None:
            raise ValueError("search takes one image and no window")
        psi, y = self._ordered(psi), self._ordered(y)
        self._run(psi, lambda a, b, mean: torch.round(y[:, a:b] - mean), step)
        start, end, C, page = int(self.bounds[step]), int(self.bounds[step + ahead]), len(offsets), self.cache.page
        per = -(-(end - start) // page)
        if C * per > len(self.spare):
            raise ValueError(f"search needs {C * per} spare pages")
        prefix, table = self.table[0, :-(-start // page)].contiguous(), self.spare[:C * per].view(C, per)
        offset = torch.tensor(offsets, dtype=torch.float32, device="cuda").view(C, 1, 1)
        error = torch.zeros(C, device="cuda")
        for a, b in zip(self.bounds[step:step + ahead].tolist(), self.bounds[step + 1:step + ahead + 1].tolist()):
            n, p = b - a, psi[:, a:b].expand(C, -1, -1)
            q = self._heads(p, self.wq, self.q_heads, a)
            seen = [torch.full((C, n), x, dtype=torch.int32, device="cuda") for x in (start, a - start)]
            ctx = self.cache.attend_shared(q, prefix, seen[0], table, seen[1], max_prefix=start, max_visible=a - start)
            mean = ctx.float().view(C, n, -1) @ self.wo + p @ self.wp
            y_hat = torch.round(y[:, a:b] - mean + offset) + mean
            self._write(y_hat, p, table, a, a - start)
            error += ((y_hat - y[:, a:b]) ** 2).sum((1, 2))
        return error

    def _ordered(self, x):
        return x.reshape(self.B, self.H * self.W, -1)[:, self.order]

    def _grid(self, x):
        out = torch.empty_like(x)
        out[:, self.order] = x
        return out.view(self.B, self.H, self.W, -1)

    def encode(self, psi, y):
        """(symbols, y_hat) [B][H][W][M] of latents y under psi [B][H][W][2M]."""
        y = self._ordered(y)
        s, y_hat = self._run(self._ordered(psi), lambda a, b, mean: torch.round(y[:, a:b] - mean))
        return self._grid(s), self._grid(y_hat)

    def decode(self, psi, symbols):
        """y_hat [B][H][W][M] from the symbols."""
        s = self._ordered(symbols)
        return self._grid(self._run(self._ordered(psi), lambda a, b, mean: s[:, a:b])[1])

    def cached(self):
        """Keys and values [B][H*W][heads][64] of the last image, as they are held."""
        first = torch.zeros(self.B, dtype=torch.int32, device="cuda")
        return self.cache.read(self.table, first, self.H * self.W)


def main():
    H, W, M = (int(x) for x in sys.argv[1:4]) if len(sys.argv) > 3 else (16, 16, 192)
    model = AttentionContext(H, W, M)
    psi = torch.from_numpy(inputs.make_psi(1, H, W, M)).cuda()
    y = 4 * torch.from_numpy(inputs.make_psi(1, H, W, M, seed=7)[..., :M].copy()).cuda()
    s, y_enc = model.encode(psi, y)
    y_dec = model.decode(psi, s)
    model.cache.sync()
    k, _ = model.cached()
    assert torch.equal(y_enc, y_dec)
    held = k.numel() * 2 * 17 / 32
    placed = AttentionContext(H, W, M, placed=True, window=4 * H, sinks=H)
    s, y_enc = placed.encode(psi, y)
    assert torch.equal(y_enc, placed.decode(psi, s))
    searching = AttentionContext(H, W, M, placed=True, spare=64)
    error = searching.search(psi, y, len(searching.bounds) // 2, 2, [-0.3, 0.0, 0.3])
    print("squared errors of three ways to round two steps:", [round(float(e), 1) for e in error])
    print(f"{H} x {W} x {M}: decoder agrees with encoder; largest |y - y_hat| {float((y - y_dec).abs().max()):.3f}; "
          f"cache {held / 1e3:.0f} kB ({k.numel() * 4 / 1e3:.0f} kB in bf16)")


if __name__ == "__main__":
    main()
