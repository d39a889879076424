"""Serving with rotary positions and a paged, quantized cache: prompts in chunks, decode steps (eager, or one captured graph replayed), a fork
that shares its pages, and a compaction.

    python examples/paged_serving.py [--layers 4 --q-heads 16 --kv-heads 4 --d 128 --bits 4 --page 16 --steps 32 --graph]

The model is as small as a model can be (per layer: q, k, v from a matrix of random weights, attention, a matrix back, added to the stream);
what is shown is the order of the calls and the bookkeeping around them, which is the caller's: Pages below.  Attention of every layer and step
is compared with plain attention over the exact keys and values, up to the first half of the decode steps; the others are timed.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


class Pages:
    """Which pages and windows each sequence has.  Full pages never change: sequences share them (counted).  A sequence has two windows,
    its tokens behind the last full page lie in one of them; a step that fills a page goes on in the other."""

    def __init__(self, n_pages: int, n_windows: int, page_tokens: int, max_pages: int):
        self.R, self.max_pages = page_tokens, max_pages
        self.free = list(range(n_pages))[::-1]               # lowest page next
        self.free_windows = list(range(n_windows))[::-1]
        self.users = [0] * n_pages
        self.pages: dict[int, list[int]] = {}
        self.length: dict[int, int] = {}
        self.windows: dict[int, list[int]] = {}              # [the one in use, the other]
        self.next_id = 0

    def add(self) -> int:
        if len(self.free_windows) < 2:
            raise RuntimeError("no window left")
        name, self.next_id = self.next_id, self.next_id + 1
        self.pages[name], self.length[name], self.windows[name] = [], 0, [self.free_windows.pop(), self.free_windows.pop()]
        return name

    def drop(self, name: int) -> None:
        for p in self.pages.pop(name):
            self.users[p] -= 1
            if self.users[p] == 0:
                self.free.append(p)
        self.free_windows += self.windows.pop(name)
        del self.length[name]

    def fork(self, name: int) -> tuple[int, tuple[int, int]]:
        """A sequence with the same tokens, and the pair of windows to copy for it."""
        new = self.add()
        self.pages[new], self.length[new] = list(self.pages[name]), self.length[name]
        for p in self.pages[new]:
            self.users[p] += 1
        return new, (self.windows[name][0], self.windows[new][0])

    def grow(self, names, new):
        """The sequences' arrays for a step that brings new[i] tokens to names[i]: page table, windows, lengths, starts (int32)."""
        need = [(self.length[n] + t) // self.R - self.length[n] // self.R for n, t in zip(names, new)]
        if sum(need) > len(self.free):
            raise RuntimeError("no page left")               # (before anything has changed)
        if any((self.length[n] + t) // self.R > self.max_pages for n, t in zip(names, new)):
            raise RuntimeError("a sequence is longer than its row of the page table")
        table, windows = np.zeros((len(names), self.max_pages), np.int32), np.zeros((len(names), 2), np.int32)
        for i, (n, t, fills) in enumerate(zip(names, new, need)):
            for _ in range(fills):
                p = self.free.pop()
                self.users[p] = 1
                self.pages[n].append(p)
            windows[i] = self.windows[n][0]
            if fills:
                self.windows[n].reverse()
                windows[i, 1] = self.windows[n][0]
            self.length[n] += t
            table[i, : len(self.pages[n])] = self.pages[n]
        starts = np.concatenate([[0], np.cumsum(new)])
        return table, windows, np.array([self.length[n] for n in names], np.int32), starts.astype(np.int32)

    def compact(self) -> list[tuple[int, int]]:
        """The pages in use to the lowest numbers: pairs (from, to), no `to` in use."""
        used = sorted(p for p, n in enumerate(self.users) if n)
        low = sorted(set(self.free))
        moves = {}
        for p in reversed(used):
            if not low or low[0] > p:
                break
            moves[p] = low.pop(0)
        for p, to in moves.items():
            self.users[to], self.users[p] = self.users[p], 0
        self.pages = {n: [moves.get(p, p) for p in ps] for n, ps in self.pages.items()}
        self.free = [p for p in range(len(self.users)) if not self.users[p]][::-1]
        return list(moves.items())


def run(layers=4, q_heads=16, kv_heads=4, d=128, bits=4, page=16, prompts=(700, 37, 1, 260), steps=24, chunk=256, graph=False, seed=0, say=print):
    """Returns the largest relative error of an attention that was compared."""
    import torch

    from paper_2605_05699_amd import binding as B

    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    steps = max(steps, 4)                                    # one after the fork, one after the compaction, then those that are compared and timed
    hidden, most = 512, max(prompts) + steps + 1
    max_seqs, max_pages = len(prompts) + 1, most // page + 1
    n_pages, n_windows = max_seqs * max_pages, 2 * max_seqs
    plans = [(B.Plan(d, 32, 2 * i + 1, None, bits), B.Plan(d, 32, 2 * i + 2, None, bits)) for i in range(layers)]
    pools = [B.PagePool.empty(*p, kv_heads, page, n_pages, n_windows) for p in plans]
    every = B.PoolTable(pools)
    heads = q_heads + 2 * kv_heads
    weights = [(torch.randn(hidden, heads * d, generator=gen, device=dev).half() / hidden ** 0.5,
                torch.randn(q_heads * d, hidden, generator=gen, device=dev).half() / (q_heads * d) ** 0.5) for _ in range(layers)]
    freq = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device=dev) / d)
    book = Pages(n_pages, n_windows, page, max_pages)
    ints = lambda a: torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device=dev)      # noqa: E731
    no_pairs = torch.zeros(0, 2, dtype=torch.int32, device=dev)
    exact: dict[int, list] = {}                              # sequence -> per layer [k, v]: what plain attention reads

    def space_for(seqs, n):
        need = max(B.srft_pool_append_workspace_bytes(pools[0], seqs, n), B.srft_pool_attention_workspace_bytes(pools[0], seqs, n, q_heads))
        return torch.empty(max(need, 1), dtype=torch.uint8, device=dev)

    def forward(x, positions, seqs, space, keep=None):
        """The layers over the step's tokens x [n, hidden]; keep(layer, q, k, v, out) sees what attention took and gave."""
        for i, (w_in, w_out) in enumerate(weights):
            qkv = (torch.nn.functional.rms_norm(x, (hidden,)) @ w_in).view(-1, heads, d)
            q, k, v = qkv[:, :q_heads], qkv[:, q_heads: q_heads + kv_heads], qkv[:, q_heads + kv_heads:]
            B.srft_rotary([(q, q), (k, k)], positions, freq)                                    # in place, both in one launch
            B.srft_pool_append(pools[i], seqs, k, v, space)
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            B.srft_pool_attention(pools[i], seqs, q, d ** -0.5, out, space)
            if keep:
                keep(i, q, k, v, out)
            x = x + out.view(-1, q_heads * d) @ w_out
        return x

    def step(names, new, keep=None):
        before = [book.length[n] for n in names]
        arrays = [ints(a) for a in book.grow(names, new)]
        seqs = B.PagedSeqs(*arrays, max_new=max(new), max_length=max(book.length[n] for n in names))
        positions = ints(np.concatenate([np.arange(b, b + t) for b, t in zip(before, new)]))
        x = torch.randn(sum(new), hidden, generator=gen, device=dev).half()
        return forward(x, positions, seqs, space_for(seqs, sum(new)), keep)

    def remember(names, new):
        """keep: the exact keys and values, and the largest relative error of the step's attention."""
        def keep(layer, q, k, v, out):
            at = 0
            for n, t in zip(names, new):
                old = exact[n][layer]
                exact[n][layer] = [torch.cat([o, y[at: at + t].float()]) for o, y in zip(old, (k, v))]
                kk, vv = [y.repeat_interleave(q_heads // kv_heads, 1).transpose(0, 1) for y in exact[n][layer]]
                s = q[at: at + t].float().transpose(0, 1) @ kk.transpose(1, 2).contiguous() * d ** -0.5
                s += torch.full(s.shape[1:], float("-inf"), device=dev).triu(s.shape[2] - t + 1)
                want = (s.softmax(-1) @ vv).transpose(0, 1)
                keep.worst = max(keep.worst, float((out[at: at + t].float() - want).norm() / want.norm()))
                at += t
        keep.worst = 0.0
        return keep

    def eager(names, new):
        keep = remember(names, new)
        step(names, new, keep)
        return keep.worst

    # prompts, all in one batch, in chunks
    names = [book.add() for _ in prompts]
    for n in names:
        exact[n] = [[torch.zeros(0, kv_heads, d, device=dev)] * 2 for _ in range(layers)]
    left, errors = list(prompts), []
    while any(left):
        new = [min(chunk, t) for t in left]
        errors.append(eager(names, new))
        left = [t - s for t, s in zip(left, new)]
    say(f"prompts of {list(prompts)} tokens: {sum(book.users)} pages, attention within {max(errors):.4f} of exact keys and values")
    # a fork: pages are shared, the window is copied, in every layer at once
    twin, pair = book.fork(names[0])
    B.srft_pool_copy(every, no_pairs, ints([pair]))
    exact[twin] = [list(kv) for kv in exact[names[0]]]
    names.append(twin)
    errors.append(eager(names, [1] * len(names)))
    say(f"a fork of sequence 0, and a step: {errors[-1]:.4f}")
    # a sequence ends, its pages come free, the others move together
    names.remove(1)
    book.drop(1)
    moves = book.compact()
    if moves:
        B.srft_pool_copy(every, ints(moves), no_pairs)
    errors.append(eager(names, [1] * len(names)))
    say(f"sequence 1 dropped, {len(moves)} pages moved, and a step: {errors[-1]:.4f}")
    # decode steps; with graph, one captured step is replayed over device arrays that are written between the replays
    new = [1] * len(names)
    if graph:
        x = torch.zeros(len(names), hidden, device=dev, dtype=torch.float16)
        arrays = [ints(a) for a in (np.zeros((len(names), max_pages)), np.zeros((len(names), 2)), np.zeros(len(names)), np.zeros(len(names) + 1))]
        positions = ints(np.zeros(len(names)))
        seqs = B.PagedSeqs(*arrays, max_new=1, max_length=most)
        space = space_for(seqs, len(names))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            forward(x, positions, seqs, space)               # (no tokens yet: nothing is stored)
        torch.cuda.current_stream().wait_stream(side)
        captured, held = torch.cuda.CUDAGraph(), []          # held: what each layer's attention takes and gives in a replay
        with torch.cuda.graph(captured):
            y = forward(x, positions, seqs, space, lambda *layer: held.append(layer))

        def decode(keep=None):
            positions.copy_(ints([book.length[n] for n in names]))
            for to, a in zip(arrays, book.grow(names, new)):
                to.copy_(ints(a))
            x.normal_(generator=gen)
            captured.replay()
            for layer in held if keep else ():
                keep(*layer)
            return y
    else:
        def decode(keep=None):
            return step(names, new, keep)
    compared = (steps - 2) // 2
    for _ in range(compared):                                # (the first replay uploads the graph, too)
        keep = remember(names, new)
        decode(keep)
        errors.append(keep.worst)
    torch.cuda.synchronize()
    start, timed = time.perf_counter(), steps - 2 - compared
    for _ in range(timed):
        decode()
    torch.cuda.synchronize()
    each = (time.perf_counter() - start) / timed
    say(f"{compared} decode steps of {len(names)} sequences, {'a captured graph' if graph else 'eager'}: {max(errors[-compared:]):.4f}; "
        f"{timed} more: {1e3 * each:.2f} ms a step")
    for p in pools:
        p.close()
    for pair in plans:
        for p in pair:
            p.close()
    return max(errors)


def main() -> int:
    p = argparse.ArgumentParser()
    for name, value in (("layers", 4), ("q-heads", 16), ("kv-heads", 4), ("d", 128), ("bits", 4), ("page", 16), ("steps", 24), ("chunk", 256)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--graph", action="store_true")
    run(**vars(p.parse_args()))
    return 0


if __name__ == "__main__":
    sys.exit(main())
