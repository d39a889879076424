"""The example of serving over the paged cache: its bookkeeping, and the whole of it on the GPU."""
import importlib.util
from pathlib import Path

import numpy as np
import pytest

PATH = Path(__file__).resolve().parent.parent / "examples" / "paged_serving.py"


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("paged_serving", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


class Store:
    """What pages and windows hold, as the kernels would leave it: token values."""

    def __init__(self, book, pages, windows):
        self.book, self.page, self.window = book, [None] * pages, [[] for _ in range(windows)]

    def append(self, names, new, arrays, value):
        table, windows, lengths, starts = arrays
        R = self.book.R
        for i, (n, t) in enumerate(zip(names, new)):
            assert starts[i + 1] - starts[i] == t
            before = int(lengths[i]) - t
            tokens = list(self.window[windows[i, 0]][: before % R]) + [value(n, before + j) for j in range(t)]
            first = before // R
            for j in range(first, int(lengths[i]) // R):
                self.page[table[i, j]], tokens = tokens[:R], tokens[R:]
            if int(lengths[i]) // R > first:
                assert windows[i, 0] != windows[i, 1]
            else:
                assert windows[i, 0] == windows[i, 1]
            self.window[windows[i, 1]] = tokens

    def tokens(self, name):
        b = self.book
        return [x for p in b.pages[name] for x in self.page[p]] + self.window[b.windows[name][0]][: b.length[name] % b.R]


@pytest.mark.parametrize("seed", range(6))
def test_bookkeeping(example, seed):
    rng = np.random.default_rng(seed)
    n_pages, n_windows, R = 40, 16, 16
    book = example.Pages(n_pages, n_windows, R, max_pages=12)
    store, want = Store(book, n_pages, n_windows), {}
    for _ in range(200):
        act = rng.choice(["add", "grow", "grow", "grow", "fork", "drop", "compact"])
        names = sorted(book.pages)
        if act == "add" and len(names) < n_windows // 2:
            want[book.add()] = []
        elif act == "fork" and names and len(names) < n_windows // 2:
            of = int(rng.choice(names))
            new, (a, b) = book.fork(of)
            store.window[b] = list(store.window[a])
            want[new] = list(want[of])
        elif act == "drop" and names:
            gone = int(rng.choice(names))
            book.drop(gone)
            del want[gone]
        elif act == "compact":
            pairs = book.compact()
            to = [b for _, b in pairs]
            assert len(set(to)) == len(to) and not set(to) & {a for a, _ in pairs}
            copies = [(store.page[a], b) for a, b in pairs]
            for x, b in copies:
                store.page[b] = x
            used = sum(1 for u in book.users if u)
            assert all(book.users[:used]) and not any(book.users[used:])
        elif act == "grow" and names:
            some = [n for n in names if rng.random() < 0.7] or names[:1]
            new = [int(rng.integers(0, 40)) for _ in some]
            state = ([list(p) for p in book.pages.values()], dict(book.length), list(book.free))
            try:
                arrays = book.grow(some, new)
            except RuntimeError:
                assert state == ([list(p) for p in book.pages.values()], book.length, book.free)
                continue
            store.append(some, new, arrays, lambda n, j: (n, j))
            for n, t in zip(some, new):
                want[n] += [(n, book.length[n] - t + j) for j in range(t)]
        users = [0] * n_pages
        for ps in book.pages.values():
            for p in ps:
                users[p] += 1
        assert users == book.users and sorted(book.free) == [p for p in range(n_pages) if not users[p]]
        windows = [w for ws in book.windows.values() for w in ws] + book.free_windows
        assert sorted(windows) == list(range(n_windows))
        for n in book.pages:
            assert store.tokens(n) == want[n]


@pytest.mark.gpu
@pytest.mark.parametrize("bits,graph", [(8, False), (4, True)])
def test_the_example(example, bits, graph):
    """The codes' rounding against exact keys and values: half a step of a group's largest over 127 (7), uniform: 1 / 440 (1 / 24) of some
    2.2 standard deviations, for keys and for values: 0.7 % (13 %) together, and twice that for what a draw may do."""
    lines = []
    worst = example.run(layers=2, bits=bits, prompts=(150, 37, 1, 90), steps=6, chunk=64, graph=graph, say=lines.append)
    assert len(lines) == 4 and worst < 2 * (0.007 if bits == 8 else 0.13)
