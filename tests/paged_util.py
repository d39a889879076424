"""Sequences over a paged pool as a program keeps them (numpy bookkeeping), and attention over them in 64 bits with a bound on
what the kernels' roundings can do to it."""
import numpy as np
import torch

from oracle import srft_oracle as O

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


class Serving:
    """n sequences on one pool: page tables in an order of their own, two windows each, taken in turn when a page fills."""

    def __init__(self, B, d, g, bits, R, heads, n, max_length, seed, transform="dft", lam_spread=0.5, spare=3):
        self.B, self.d, self.g, self.bits, self.R, self.heads, self.n = B, d, g, bits, R, heads, n
        self.rng, self.transform = np.random.default_rng(seed), transform
        self.lam = [np.exp(lam_spread * self.rng.standard_normal(d)).astype(np.float32) for _ in range(2)]
        self.plans = [B.Plan(d, g, seed + i, self.lam[i], bits, transform) for i in range(2)]
        self.max_pages = max(1, max_length // R)
        pages = n * self.max_pages + spare
        self.pool = B.PagePool.empty(*self.plans, heads, R, pages, 2 * n + 1)
        for _, s, w in (self.pool.k, self.pool.v):           # what nobody has written is not a number
            s.fill_(float("nan"))
            w.fill_(float("nan"))
        self.free = list(self.rng.permutation(pages))
        self.table = np.full((n, self.max_pages), -1, np.int32)
        self.slots = self.rng.permutation(2 * n + 1)[: 2 * n].reshape(n, 2).astype(np.int32)
        self.windows = np.stack([self.slots[:, 0]] * 2, 1)
        self.length = np.zeros(n, np.int64)
        self.max_length = max_length
        self.tokens = [[np.zeros((0, heads, d), np.float16) for _ in range(n)] for _ in range(2)]
        self.workspace = None

    def seqs(self, new, **bounds):
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        to = lambda a: torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")      # noqa: E731
        return self.B.PagedSeqs(to(self.table), to(self.windows), to(self.length), to(starts), **{"max_new": int(max(new)), "max_length": self.max_length, **bounds})

    def grow(self, new):
        """Lengths, page tables and windows of the sequences after new[b] more tokens."""
        for b, t in enumerate(new):
            before, after = self.length[b] // self.R, (self.length[b] + t) // self.R
            for j in range(before, after):
                self.table[b, j] = self.free.pop()
            self.windows[b, 0] = self.windows[b, 1]
            if after > before:
                self.windows[b, 1] = self.slots[b, 0] + self.slots[b, 1] - self.windows[b, 1]
            self.length[b] += t

    def draw(self, n, gain=1.0):
        x = self.rng.standard_normal((n, self.heads, self.d))
        x[..., self.d // 3] *= 10.0
        return (gain * x).astype(np.float16)

    def append(self, new, gain=1.0, stream=None):
        kv = [self.draw(int(sum(new)), gain) for _ in range(2)]
        self.grow(new)
        at = 0
        for b, t in enumerate(new):
            for i in range(2):
                self.tokens[i][b] = np.concatenate([self.tokens[i][b], kv[i][at: at + t]])
            at += t
        seqs = self.seqs(new)
        dev = [torch.from_numpy(x).cuda() for x in kv]
        space = torch.empty(self.B.srft_pool_append_workspace_bytes(self.pool, seqs, int(sum(new))), dtype=torch.uint8, device="cuda")
        self.B.srft_pool_append(self.pool, seqs, *dev, space, stream)
        return seqs

    def stored(self, which, b, pages=None):
        """(codes, scales) of sequence b's full pages, [tokens, heads, ...] (numpy)."""
        codes, scales, _ = self.pool.k if which == 0 else self.pool.v
        ids = torch.tensor(self.table[b, : self.length[b] // self.R].astype(np.int64), device="cuda")
        return tuple(t[ids].permute(0, 2, 1, 3).flatten(0, 1).cpu().numpy() for t in (codes, scales))

    def window(self, which, b):
        return (self.pool.k if which == 0 else self.pool.v)[2][int(self.windows[b, 1])].permute(1, 0, 2).cpu().numpy()

    def values(self, which, b):
        """What attention sees, in the rotated domain (w = lambda * pack(F (s * x))), fp64 [length, heads, d]."""
        codes, scales = self.stored(which, b)
        full = self.length[b] // self.R * self.R
        if self.bits == 8:
            q = codes.view(np.int8).astype(np.float64)
        else:
            low = lambda x: ((x.astype(np.int64) & 15) ^ 8) - 8      # noqa: E731
            q = np.stack([low(codes), low(codes >> 4)], -1).reshape(*codes.shape[:-1], self.d).astype(np.float64)
        w = q * np.repeat(scales.astype(np.float64), self.d // scales.shape[-1], -1)
        tail = self.window(which, b)[: self.length[b] - full].astype(np.float64) @ self.matrix(which).T
        return np.concatenate([w, tail])

    def matrix(self, which):
        """W with w = W x."""
        return self.lam[which].astype(np.float64)[:, None] * self.Q() * np.asarray(self.plans[which].signs, np.float64)

    def inverse(self, which):
        """R with x = R w."""
        return (self.Q() * np.asarray(self.plans[which].signs, np.float64)).T / np.maximum(self.lam[which].astype(np.float64), 1e-6)

    def Q(self):
        return O.hadamard_matrix(self.d) if self.transform == "hadamard" else O.srft_matrix(self.d)

    def attention(self, q, new, scale, group, step, there=None, hidden=None):
        """(out, bound) for q [n_new, heads * group, d] (fp64 values): the definition, and how far a kernel may be from it that rounds
        q', code scales, dequantized codes and weights to fp16 and the result with half a step of `step`.  there[b]: mask of the tokens
        that exist.  hidden(rows' tokens, tokens): what rows do not see although it is theirs."""
        out, err = np.zeros(q.shape), np.zeros(q.shape)
        rk, rv, u, at = self.inverse(0), self.inverse(1), 2.0 ** -11, 0
        for b, t in enumerate(new):
            wk, wv = self.values(0, b), self.values(1, b)
            n = int(self.length[b])
            for h in range(self.heads):
                rows = q[at: at + t, h * group: (h + 1) * group].reshape(-1, self.d)
                limit = np.repeat(np.arange(n - t, n), group)
                see = np.arange(n)[None] <= limit[:, None]
                if hidden is not None:
                    see &= ~hidden(limit[:, None], np.arange(n)[None])
                if there is not None:
                    see &= there[b][None, :n]
                k, v = np.where(np.isfinite(wk[:, h]), wk[:, h], 0.0), np.where(np.isfinite(wv[:, h]), wv[:, h], 0.0)
                rot = rows @ rk
                s = np.where(see, scale * (rot @ k.T), -np.inf)
                # a score: three roundings of each product, and its sum in 32 bits
                ds = abs(scale) * (np.abs(rot) @ np.abs(k).T) * (3 * u * 1.01 + self.d * 2.0 ** -23) + 2.0 ** -22 * np.abs(np.where(see, s, 0.0))
                top = np.where(see.any(1), s.max(1, initial=-np.inf), 0.0)
                p = np.where(see, np.exp(s - top[:, None]), 0.0)
                den = np.maximum(p.sum(1, keepdims=True), 1e-300)
                p = p / den
                mean = (p * ds).sum(1, keepdims=True)
                rel = 1.05 * (ds + mean) + 3 * u * 1.01 + n * 2.0 ** -23
                o = (p @ v) @ rv.T
                # (fp16 weights below 2^-14 are off by up to 2^-25; the last product and its operands in 21 bits; fp16 results below 2^-14)
                small = see.sum(1, keepdims=True) * 2.0 ** -25 * np.abs(v).max(0, initial=0.0)
                e = ((p * rel) @ np.abs(v) + small + 2.0 ** -20 * (p @ np.abs(v))) @ np.abs(rv).T + step * np.abs(o) * 1.01 + 2.0 ** -25
                out[at: at + t, h * group: (h + 1) * group] = o.reshape(t, group, self.d)
                err[at: at + t, h * group: (h + 1) * group] = e.reshape(t, group, self.d)
            at += t
        return out, err

    def run(self, q, new, scale, out=None, seqs=None, stream=None):
        seqs = seqs or self.seqs(new)
        out = torch.full_like(q, float("nan")) if out is None else out
        need = self.B.srft_pool_attention_workspace_bytes(self.pool, seqs, q.shape[0], q.shape[1])
        space = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        self.B.srft_pool_attention(self.pool, seqs, q, scale, out, space, stream)
        return out

    def close(self):
        torch.cuda.synchronize()
        self.pool.close()
        for p in self.plans:
            p.close()
