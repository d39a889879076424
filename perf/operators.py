"""The operators of a serving step over a paged cache: what is timed of them, in elementary torch and through the library.

  rotary     rotary positions on queries and keys in one call: ``srft_rotary``
  append     new tokens of ragged sequences into the pages of a quantized cache: ``srft_pool_append``
  attention  causal attention of new tokens (one each, or a chunk) over the pages: ``srft_pool_attention``
  copy       pages and windows copied within the pools of several layers (fork, compaction): ``srft_pool_copy``

The cache of one layer is a pool of pages for K and one for V.  A page holds ``page`` tokens of ``kv_heads`` heads as the
quantizer's record (codes, fp32 scales); a sequence's last ``len % page`` tokens are exact fp16 in a window.  A record is
``code * scale`` in the packed transform domain: x = S Q^T diag(1 / lambda) (code * scale), with Q the real packing of the
unitary DFT and S a diagonal of signs.

Sequence b of a call brings the rows ``starts[b] .. starts[b + 1]`` of the new tokens and holds ``lengths[b]`` tokens with
them; its token j lies in page ``table[b][j / page]``, or in the window ``windows[b][1]`` if it is behind the last full page
(``windows[b][0]`` is the window that it had before the call).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------- cases
def listed() -> list[dict]:
    rot = dict(op="rotary", d=128, rot=128, layout="half", x="f16", y="f16", inverse=False, far=32768, stretch=1.0)
    page = dict(d=128, g=32, bits=4, page=16)
    app = dict(page, op="append")
    att = dict(page, op="attention", q="f16")
    return [
        # a decode step of 8 sequences, 12 query heads and 2 key heads: all latency
        dict(rot, name="rotary_step", tokens=8, q_heads=12, kv_heads=2),
        # a prompt of 8192 tokens in bf16, 32 + 8 heads, keys and queries to fp16, positions stretched for a long context
        dict(rot, name="rotary_prompt", tokens=8192, q_heads=32, kv_heads=8, x="bf16", far=131072, stretch=8.0),
        # the gradient of a training batch: fp32, interleaved pairs, the first 64 of 96 channels, an odd number of tokens
        dict(rot, name="rotary_grad", tokens=5003, q_heads=24, kv_heads=24, d=96, rot=64, layout="pairs", x="f32", y="f32",
             inverse=True),
        # a decode step of 64 sequences: a window's worth of them fill a page
        dict(app, name="append_step", seqs=64, len_min=1, len_max=4000, new_min=1, new_max=1, kv_heads=8),
        # prompts of 300 to 3000 tokens, ragged, in one call
        dict(app, name="append_prompts", seqs=12, len_min=300, len_max=3000, new_min=300, new_max=3000, kv_heads=8),
        # chunks at d = 256 with 8-bit codes, on top of prefixes that end inside a page
        dict(app, name="append_chunks_d256", seqs=6, len_min=1500, len_max=4001, new_min=200, new_max=1000, kv_heads=4, d=256,
             bits=8, page=64),
        # one decode step of 4 short sequences, 6 query heads to a key head
        dict(att, name="decode_short", seqs=4, len_min=60, len_max=1000, new_min=1, new_max=1, kv_heads=2, group=6),
        # one decode step of a serving batch: 24 ragged sequences up to 32768 tokens, 64 query and 8 key heads
        dict(att, name="decode_batch", seqs=24, len_min=500, len_max=32768, new_min=1, new_max=1, kv_heads=8, group=8),
        # a chunk of a long prompt behind the tokens that the cache has already, 32 query and 8 key heads
        dict(att, name="chunk_long", seqs=1, len_min=16384, len_max=16384, new_min=2048, new_max=2048, kv_heads=8, group=4),
        # two prompts' chunks and decode steps in one batch, d = 256 with 8-bit codes, pages of 64, bf16 queries
        dict(att, name="mixed_d256", seqs=8, len_min=700, len_max=4096, new_min=1, new_max=500, kv_heads=4, group=2, d=256, bits=8,
             page=64, q="bf16"),
        # a fork: a few pages and every layer's windows
        dict(page, op="copy", name="copy_fork", layers=8, kv_heads=2, pages=3, windows=4, pool=64),
        # compaction: many pages of many layers move down
        dict(page, op="copy", name="copy_compact", layers=16, kv_heads=8, pages=1500, windows=0, pool=4096),
    ]


def _log_int(rng: random.Random, lo: float, hi: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random) -> dict:
    op = rng.choice(["rotary", "append", "attention", "attention", "attention", "copy"])
    kv = rng.choice([1, 2, 3, 4, 8])
    if op == "rotary":
        d = rng.choice([64, 96, 128, 192, 256])
        x = rng.choice(["f16", "bf16", "f32"])
        return dict(op=op, tokens=_log_int(rng, 1, 8192), q_heads=kv * rng.choice([1, 3, 4]), kv_heads=kv, d=d,
                    rot=rng.choice([d, d // 2, 32]), layout=rng.choice(["half", "pairs"]), x=x, y=rng.choice([x, "f16"]),
                    inverse=rng.random() < 0.4, far=_log_int(rng, 2048, 1000000), stretch=rng.choice([1.0, 1.0, 4.0, 32.0]))
    d = rng.choice([64, 96, 128, 128, 128, 192, 256])
    page = rng.choice([16, 32, 64, 128])
    if kv % 2 and page == 16:
        page = 32
    shape = dict(d=d, g=rng.choice([32, 32, 32, 16, d]), bits=rng.choice([4, 4, 8]), page=page)
    if op == "copy":
        layers = rng.choice([1, 4, 16])
        return dict(shape, op=op, layers=layers, kv_heads=kv, pages=_log_int(rng, 1, 200), windows=rng.randrange(0, 5), pool=512)
    if op == "append":
        seqs, new = rng.randint(1, 40), rng.choice([1, 1, _log_int(rng, 2, 700)])
        # (as many new tokens as fill at most one page, or a prompt from its first token on: the call can be made again)
        if new < page:                                       # (mostly into a window; else prompts and chunks)
            return dict(shape, op=op, seqs=seqs, len_min=new + rng.randrange(0, 300), len_max=new + 300 + rng.randrange(0, 3000),
                        new_min=max(1, new // 2), new_max=new, kv_heads=kv)
        return dict(shape, op=op, seqs=seqs, len_min=max(1, new // 4), len_max=new + rng.choice([0, 500]), new_min=max(1, new // 4), new_max=new, kv_heads=kv)
    group = rng.choice([1, 2, 4, 6, 8])
    kind = rng.choice(["decode", "decode", "chunk", "mixed"])
    if kind == "decode":
        seqs, top, new = _log_int(rng, 1, 32), _log_int(rng, 50, 16000), rng.choice([1, 1, 1, 4])
        lo = max(1, int(top * rng.uniform(0.02, 1.0)))
        return dict(shape, op="attention", q=rng.choice(["f16", "bf16"]), seqs=seqs, len_min=min(lo, top), len_max=top, new_min=1,
                    new_max=new, kv_heads=kv, group=group)
    seqs = rng.randint(1, 3) if kind == "chunk" else rng.randint(3, 8)
    new = _log_int(rng, 20, 800)
    top = new + _log_int(rng, 1, 5000)
    return dict(shape, op="attention", q=rng.choice(["f16", "bf16"]), seqs=seqs, len_min=max(1, top // rng.choice([1, 2, 8])),
                len_max=top, new_min=new if kind == "chunk" else 1, new_max=new, kv_heads=kv, group=group)


def _ragged(case: dict) -> tuple[np.ndarray, np.ndarray]:
    """(lengths with the new tokens, new tokens) of a case's sequences: spread over their ranges, odd ones among them."""
    n = case["seqs"]
    at = (np.arange(n) * 7 % n + 0.5) / n if n % 7 else (np.arange(n) + 0.5) / n
    at[0] = 1.0
    lens = np.rint(case["len_min"] + (case["len_max"] - case["len_min"]) * at ** 2).astype(np.int64)
    new = np.rint(case["new_min"] + (case["new_max"] - case["new_min"]) * (at if case["new_min"] * 4 > case["new_max"] else at ** 4))
    return lens, np.minimum(new.astype(np.int64), lens)


# ----------------------------------------------------------------------------------------------------- the record's constants
def _signs(seed: int, d: int) -> np.ndarray:
    """splitmix64 from `seed`: -1 where the top bit of the n-th output is set."""
    mask, state, out = (1 << 64) - 1, seed & ((1 << 64) - 1), np.empty(d)
    for n in range(d):
        state = (state + 0x9E3779B97F4A7C15) & mask
        z = ((state ^ (state >> 30)) * 0xBF58476D1CE4E5B9) & mask
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
        out[n] = -1.0 if (z ^ (z >> 31)) >> 63 else 1.0
    return out


def _constants(seed: int, d: int) -> tuple[np.ndarray, np.ndarray, np.ndarray]:
    """(lambda as fp32, W with w = W x, R with x = R w) of one of K and V."""
    lam = np.exp(0.5 * np.random.RandomState(seed % (1 << 32)).standard_normal(d)).astype(np.float32)
    k, n = np.arange(d // 2 + 1)[:, None], np.arange(d)[None, :]
    angle = 2.0 * np.pi * (k * n % d) / d
    q = np.empty((d, d))
    q[: d // 2 + 1] = np.cos(angle) * math.sqrt(2.0 / d)
    q[d // 2 + 1:] = -np.sin(angle[1: d // 2]) * math.sqrt(2.0 / d)
    q[0] /= math.sqrt(2.0)
    q[d // 2] /= math.sqrt(2.0)
    s, wide = _signs(seed, d), lam.astype(np.float64)
    return lam, wide[:, None] * q * s, (q * s).T / np.maximum(wide, 1e-6)


def _quantize(x: torch.Tensor, w: torch.Tensor, g: int, bits: int) -> tuple[torch.Tensor, torch.Tensor]:
    """The write path in plain operations: rows x -> (codes as stored, scales)."""
    top = 7.0 if bits == 4 else 127.0
    y = (x.float() @ w.T).unflatten(-1, (-1, g))
    scale = y.abs().amax(-1) / top
    code = torch.round(y / torch.where(scale > 0, scale, 1.0)[..., None]).to(torch.int16).flatten(-2)
    if bits == 8:
        return code.to(torch.int8).view(torch.uint8), scale
    return ((code[..., 0::2] & 15) | ((code[..., 1::2] & 15) << 4)).to(torch.uint8), scale


def _values(codes: torch.Tensor, scales: torch.Tensor, bits: int) -> torch.Tensor:
    """code * scale of stored rows, in the scales' type."""
    if bits == 8:
        q = codes.view(torch.int8).to(scales.dtype)
    else:
        wide = codes.to(torch.int16)
        q = torch.stack([((wide & 15) ^ 8) - 8, (wide >> 4 ^ 8) - 8], -1).flatten(-2).to(scales.dtype)
    return (q.unflatten(-1, (scales.shape[-1], -1)) * scales[..., None]).flatten(-2)


# ------------------------------------------------------------------------------------------------------------------ inputs
def _rows(gen: torch.Generator, shape: tuple, outlier: bool) -> torch.Tensor:
    x = torch.randn(*shape, device=DEVICE, generator=gen, dtype=torch.float16)
    if outlier:
        x[..., shape[-1] // 3] *= 10.0                       # K: one persistent outlier channel
    return x


def _frequencies(case: dict) -> np.ndarray:
    """Radians a token of each pair: base 10000, the slow half of them stretched."""
    f = 10000.0 ** (-np.arange(0, case["rot"], 2) / case["rot"])
    f[len(f) // 2:] /= case["stretch"]
    return f


def _prepare_rotary(case: dict, gen: torch.Generator) -> dict:
    n, h, d = case["tokens"], case["q_heads"] + 2 * case["kv_heads"], case["d"]
    packed = torch.randn(n, h, d, device=DEVICE, generator=gen).to(DTYPES[case["x"]])      # q, k and v next to each other
    st = {"q": packed[:, : case["q_heads"]], "k": packed[:, case["q_heads"]: case["q_heads"] + case["kv_heads"]],
          "q_out": torch.empty(n, case["q_heads"], d, device=DEVICE, dtype=DTYPES[case["y"]]),
          "k_out": torch.empty(n, case["kv_heads"], d, device=DEVICE, dtype=DTYPES[case["y"]]),
          "positions": torch.randint(0, case["far"], (n,), device=DEVICE, generator=gen, dtype=torch.int32),
          "freq": torch.tensor(_frequencies(case), device=DEVICE), "factor": 1.0 + 0.1 * math.log(case["stretch"])}
    return st


def _plan_seeds(seed: int) -> tuple[int, int]:
    return seed * 1_000_003 + 1, seed * 1_000_003 + 2


def _prepare_pages(case: dict, seed: int, gen: torch.Generator) -> dict:
    d, g, bits, page, heads = (case[k] for k in ("d", "g", "bits", "page", "kv_heads"))
    lens, new = _ragged(case)
    before = lens - new if case["op"] == "append" else lens
    n = len(lens)
    full, had = lens // page, before // page
    rng = np.random.RandomState(seed % (1 << 32))
    # pages that this call fills come first in the pool, the others behind them, each in an order of its own
    fills, others = int((full - had).sum()), int(had.sum())
    first, rest = rng.permutation(fills), fills + rng.permutation(others)
    table = np.full((n, int(full.max()) + 1), -1, np.int32)
    for b in range(n):
        table[b, : had[b]], rest = rest[: had[b]], rest[had[b]:]
        table[b, had[b]: full[b]], first = first[: full[b] - had[b]], first[full[b] - had[b]:]
    slots = rng.permutation(2 * n).reshape(n, 2).astype(np.int32)
    slots[:, 1] = np.where(full > had, slots[:, 1], slots[:, 0])
    st = {"lens": lens, "new": new, "fills": fills, "max_new": int(new.max()), "max_len": int(lens.max()),
          "table": torch.tensor(table, device=DEVICE), "windows": torch.tensor(slots, device=DEVICE),
          "lengths": torch.tensor(lens.astype(np.int32), device=DEVICE),
          "starts": torch.tensor(np.concatenate([[0], np.cumsum(new)]).astype(np.int32), device=DEVICE)}
    for name, plan_seed in zip("kv", _plan_seeds(seed)):
        lam, w, r = _constants(plan_seed, d)
        w32 = torch.tensor(w, device=DEVICE, dtype=torch.float32)
        codes = torch.zeros(fills + others, heads, page, d * bits // 8, device=DEVICE, dtype=torch.uint8)
        scales = torch.zeros(fills + others, heads, page, d // g, device=DEVICE)
        for at in range(fills, fills + others, 4096):
            m = min(4096, fills + others - at)
            codes[at: at + m], scales[at: at + m] = _quantize(_rows(gen, (m, heads, page, d), name == "k"), w32, g, bits)
        st[name] = {"seed": plan_seed, "lam": lam, "w": w32, "r": torch.tensor(r, device=DEVICE, dtype=torch.float32), "codes": codes,
                    "scales": scales, "window": _rows(gen, (2 * n, heads, page, d), name == "k")}
    return st


def _pool(case: dict, k: dict, v: dict):
    """The library's handle of one layer's pages, over the tensors of the state."""
    from paper_2605_05699_amd import binding as B
    plans = [B.Plan(case["d"], case["g"], s["seed"], s["lam"], bits=case["bits"]) for s in (k, v)]
    return B.PagePool(*plans, *[(s["codes"], s["scales"], s["window"]) for s in (k, v)])


def _keep(case: dict, st: dict) -> None:
    """What a program keeps between steps beside its buffers: the handle, the batch's description and a workspace."""
    from paper_2605_05699_amd import binding as B
    st["pool"] = _pool(case, st["k"], st["v"])
    st["seqs"] = B.PagedSeqs(st["table"], st["windows"], st["lengths"], st["starts"], max_new=st["max_new"], max_length=st["max_len"])
    if case["op"] == "append":
        size = B.srft_pool_append_workspace_bytes(st["pool"], st["seqs"], int(st["new"].sum()))
        k, v = st["k"], st["v"]
        n, d = st["fills"] * case["kv_heads"] * case["page"], case["d"]
        if n:
            st["back"] = [torch.empty(n, d, device=DEVICE, dtype=torch.float16) for _ in "kv"]
            st["read"] = B.BatchTable([p.handle for p in st["pool"].plans], st["back"], [s["codes"].view(-1, s["codes"].shape[-1])[:n] for s in (k, v)],
                                      [s["scales"].view(-1, s["scales"].shape[-1])[:n] for s in (k, v)])
    else:
        size = B.srft_pool_attention_workspace_bytes(st["pool"], st["seqs"], st["q"].shape[0], st["q"].shape[1])
    st["workspace"] = torch.empty(size, device=DEVICE, dtype=torch.uint8)


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(DEVICE)
    gen.manual_seed(seed)
    if case["op"] == "rotary":
        st = _prepare_rotary(case, gen)
    elif case["op"] == "copy":
        st = _prepare_copy(case, seed, gen)
    else:
        st = _prepare_pages(case, seed, gen)
        n, d = int(st["new"].sum()), case["d"]
        if case["op"] == "append":
            st["k_new"], st["v_new"] = (_rows(gen, (n, case["kv_heads"], d), name == "k") for name in "kv")
        else:
            st["q"] = torch.randn(n, case["kv_heads"] * case["group"], d, device=DEVICE, generator=gen).to(DTYPES[case["q"]])
            st["out"] = torch.empty_like(st["q"])
            st["scale"] = d ** -0.5
        if own:
            _keep(case, st)
    st["case"] = case
    return st


def _prepare_copy(case: dict, seed: int, gen: torch.Generator) -> dict:
    d, g, bits, page, heads, layers, size = (case[k] for k in ("d", "g", "bits", "page", "kv_heads", "layers", "pool"))
    rng = np.random.RandomState(seed % (1 << 32))
    at, win = rng.permutation(size)[: 2 * case["pages"]].reshape(-1, 2), rng.permutation(16)[: 2 * case["windows"]].reshape(-1, 2)
    st = {"pages": torch.tensor(at.astype(np.int32), device=DEVICE), "wins": torch.tensor(win.astype(np.int32), device=DEVICE)}
    for name, plan_seed in zip("kv", _plan_seeds(seed)):
        st[name] = {"seed": plan_seed, "lam": _constants(plan_seed, d)[0],
                    "codes": torch.randint(0, 256, (layers, size, heads, page, d * bits // 8), device=DEVICE, generator=gen, dtype=torch.uint8),
                    "scales": torch.rand(layers, size, heads, page, d // g, device=DEVICE, generator=gen),
                    "window": torch.randn(layers, 16, heads, page, d, device=DEVICE, generator=gen, dtype=torch.float16)}
    if own:
        from paper_2605_05699_amd import binding as B
        layer = [[{**st[x], **{f: st[x][f][i] for f in ("codes", "scales", "window")}} for x in "kv"] for i in range(layers)]
        st["pools"] = B.PoolTable([_pool(case, *kv) for kv in layer])
    return st


# --------------------------------------------------------------------------------------------------- the plain forms, and ours
def _rotate(st: dict, x: torch.Tensor, y: torch.dtype) -> torch.Tensor:
    case, rot = st["case"], st["case"]["rot"]
    angle = st["positions"].double()[:, None, None] * st["freq"]             # (64 bits: far positions)
    cos, sin = (torch.cos(angle) * st["factor"]).float(), (torch.sin(angle) * st["factor"]).float()
    if case["inverse"]:
        sin = -sin
    part, rest = x[..., :rot].float(), x[..., rot:].float()
    a, b = (part[..., : rot // 2], part[..., rot // 2:]) if case["layout"] == "half" else (part[..., 0::2], part[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([u, v], -1) if case["layout"] == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([turned, rest], -1).to(y)


def _plain_append(st: dict) -> list[torch.Tensor]:
    case = st["case"]
    page, n = case["page"], st["k_new"].shape[0]
    row = torch.arange(n, device=DEVICE)
    seq = torch.searchsorted(st["starts"], row, right=True, out_int32=True).long() - 1
    lengths = st["lengths"].long()
    before = lengths - (st["starts"][1:] - st["starts"][:-1]).long()
    pos = before[seq] + row - st["starts"].long()[seq]
    full = lengths // page
    # where the tokens of the filled pages come from: a row of [windows' tokens, new tokens] for each (page, slot)
    fills, slots = st["fills"], st["windows"].shape[0] * 2
    source = torch.zeros(fills + 1, page, device=DEVICE, dtype=torch.long)
    at = torch.where(pos // page < full[seq], st["table"].long()[seq, pos // page], fills)     # (the others go to a page that nobody reads)
    source[at, pos % page] = slots * page + row
    j = torch.arange(page, device=DEVICE)[None]
    held = (j < (before % page)[:, None]) & (full > before // page)[:, None]
    at = torch.where(held, st["table"].long().gather(1, (before // page)[:, None]), fills)
    kept = st["windows"][:, :1].long() * page + j
    source[at, j.expand_as(at)] = torch.where(held, kept, source[at, j.expand_as(at)])
    # what is behind a sequence's last full page: slot j of its window is the row starts[b + 1] - len % page + j, if that is new
    tail = (lengths % page)[:, None]
    behind = (st["starts"][1:].long()[:, None] - tail + j).clamp(0, n - 1)
    fresh = (j < tail) & (j >= tail - (lengths - before)[:, None])
    out = []
    for name, new in (("k", st["k_new"]), ("v", st["v_new"])):
        s = st[name]
        rows = torch.cat([s["window"].transpose(1, 2).flatten(0, 1), new])
        codes, scales = _quantize(rows[source[:fills]].transpose(1, 2), s["w"], case["g"], case["bits"])
        s["codes"][:fills], s["scales"][:fills] = codes, scales
        to = st["windows"][:, 1].long()
        s["window"][to] = torch.where(fresh[:, None, :, None], new[behind].transpose(1, 2), s["window"][to])
        out += [(_values(codes, scales, case["bits"]) @ s["r"].T).half().flatten(0, 2), s["window"]]
    return out


def _plain_attention(st: dict) -> torch.Tensor:
    case = st["case"]
    page, d, heads, group = (case[k] for k in ("page", "d", "kv_heads", "group"))
    lengths, starts = st["lengths"].long(), st["starts"].long()
    n_seq, most = len(lengths), st["max_len"] // page
    full = lengths // page * page
    table = st["table"][:, :most].clamp(min=0).long()
    kv = []
    for name in "kv":
        s = st[name]
        held = (_values(s["codes"][table], s["scales"][table], case["bits"]) @ s["r"].T).transpose(1, 2).flatten(2, 3)
        kv.append(torch.cat([held, s["window"][st["windows"][:, 1].long()].float()], 2))       # [seq, head, token, d]
    j = torch.arange(most * page, device=DEVICE)[None]
    behind = full[:, None] + torch.arange(page, device=DEVICE)[None]
    pos = torch.cat([torch.where(j < full[:, None], j, 1 << 40), torch.where(behind < lengths[:, None], behind, 1 << 40)], 1)
    new = starts[1:] - starts[:-1]
    i = torch.arange(st["max_new"], device=DEVICE)[None]
    row = (starts[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)
    limit = torch.where(i < new[:, None], (lengths - new)[:, None] + i, -1)
    q = st["q"].float()[row].unflatten(2, (heads, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)      # [seq, head, token * group, d]
    s = torch.matmul(q, kv[0].transpose(2, 3).contiguous()).unflatten(2, (-1, group)) * st["scale"]
    s = torch.where((pos[:, None, :] <= limit[:, :, None])[:, None, :, None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), kv[1]).unflatten(2, (-1, group)) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 2, 1, 3, 4).flatten(2, 3)                                                # [seq, token, query head, d]
    r = torch.arange(st["q"].shape[0], device=DEVICE)
    seq = torch.searchsorted(starts, r, right=True) - 1
    return o[seq, r - starts[seq]].to(st["q"].dtype)


def run(state: dict):
    op = state["case"]["op"]
    if own:
        from paper_2605_05699_amd import binding as B
        if op == "rotary":
            B.srft_rotary([(state["q"], state["q_out"]), (state["k"], state["k_out"])], state["positions"], state["freq"], layout=state["case"]["layout"],
                          factor=state["factor"], inverse=state["case"]["inverse"])
            return [state["q_out"], state["k_out"]]
        if op == "append":
            B.srft_pool_append(state["pool"], state["seqs"], state["k_new"], state["v_new"], state["workspace"])
            back = []
            if state["fills"]:                               # what the filled pages hold, through the read path
                B.srft_kv_dequantize_batched(state["read"])
                back = state["back"]
            return [x for i, s in enumerate("kv") for x in (back[i: i + 1] + [state[s]["window"]])]
        if op == "attention":
            B.srft_pool_attention(state["pool"], state["seqs"], state["q"], state["scale"], state["out"], state["workspace"])
            return state["out"]
        B.srft_pool_copy(state["pools"], state["pages"], state["wins"])
        return [state[s][f] for s in "kv" for f in ("codes", "scales", "window")]
    if op == "rotary":
        return [_rotate(state, state[x], state[x + "_out"].dtype) for x in "qk"]
    if op == "append":
        got = _plain_append(state)
        return got if state["fills"] else got[1::2]
    if op == "attention":
        return _plain_attention(state)
    for s in (state["k"], state["v"]):
        for f, at in (("codes", state["pages"]), ("scales", state["pages"]), ("window", state["wins"])):
            s[f][:, at[:, 1].long()] = s[f][:, at[:, 0].long()]
    return [state[s][f] for s in "kv" for f in ("codes", "scales", "window")]


# ------------------------------------------------------------------------------------------------------------------- the work
def work(case: dict) -> dict:
    d = case["d"]
    if case["op"] == "rotary":
        n = case["tokens"] * (case["q_heads"] + case["kv_heads"])
        size = {"f16": 2, "bf16": 2, "f32": 4}
        return {"bytes": n * d * (size[case["x"]] + size[case["y"]]) + 4 * case["tokens"], "flops": 3 * n * case["rot"]}
    heads, page = case["kv_heads"], case["page"]
    record = d * case["bits"] // 8 + 4 * (d // case["g"])
    if case["op"] == "copy":
        return {"bytes": 4 * case["layers"] * heads * page * (case["pages"] * record + case["windows"] * 2 * d), "flops": 0}
    lens, new = _ragged(case)
    full, had = lens // page, (lens - new) // page
    if case["op"] == "append":
        rows = heads * page * int((full - had).sum())
        held = heads * int(((lens - new) % page * (full > had)).sum())
        tail = heads * int(np.minimum(lens - full * page, new).sum())
        # the new tokens and those that the windows held of filled pages, the record, the windows, and the record read back to fp16
        return {"bytes": 2 * (heads * int(new.sum()) * 2 * d + held * 2 * d + rows * record + tail * 2 * d + rows * (record + 2 * d)),
                "flops": 2 * 2 * rows * 5 * d * math.log2(d)}
    rows = heads * case["group"] * int(new.sum())
    pairs = heads * case["group"] * int(sum(n * (m - n) + n * (n + 1) // 2 for m, n in zip(lens.tolist(), new.tolist())))
    return {"bytes": 2 * heads * int((full * page * record + (lens - full * page) * 2 * d).sum()) + 2 * rows * 2 * d, "flops": 4 * pairs * d}


# --------------------------------------------------------------------------------------------------- by definition, in 64 bits
def _decoded(codes: torch.Tensor, scales: torch.Tensor, bits: int) -> torch.Tensor:
    """Stored rows in 64 bits: what each byte stands for is looked up."""
    low = [(i & 15) - 16 * (i >> 3 & 1) for i in range(256)]
    pair = [(a, low[i >> 4]) for i, a in enumerate(low)] if bits == 4 else [(i - 256 * (i >> 7),) for i in range(256)]
    q = torch.tensor(pair, device=DEVICE, dtype=torch.float64)[codes.long()].flatten(-2)
    return q * scales.double().repeat_interleave(q.shape[-1] // scales.shape[-1], -1)


def exact(case: dict, seed: int):
    state = prepare(case, seed)
    if case["op"] == "rotary":
        f = _frequencies(case)
        z = torch.polar(torch.full((case["tokens"], len(f)), 1.0 + 0.1 * math.log(case["stretch"]), device=DEVICE, dtype=torch.float64),
                        state["positions"].double()[:, None] * torch.tensor(f, device=DEVICE))
        z = z.conj() if case["inverse"] else z
        out = []
        for x in (state["q"], state["k"]):
            y, r = x.double().clone(), case["rot"]
            first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
            t = torch.complex(y[..., first], y[..., second]) * z[:, None]
            y[..., first], y[..., second] = t.real, t.imag
            out.append(y)
        return out
    if case["op"] == "copy":
        return None
    lens, new = state["lens"].tolist(), state["new"].tolist()
    table, wins, page, bits = state["table"].cpu().numpy(), state["windows"].cpu().numpy(), case["page"], case["bits"]
    back = {s: torch.tensor(_constants(state[s]["seed"], case["d"])[2], device=DEVICE) for s in "kv"}
    if case["op"] == "append":
        if case["seqs"] * case["new_max"] > 40000:
            return None
        out = []
        for s, x in (("k", state["k_new"]), ("v", state["v_new"])):
            forward, steps = torch.tensor(_constants(state[s]["seed"], case["d"])[1], device=DEVICE), 7.0 if bits == 4 else 127.0
            window, pages, at = state[s]["window"].double(), torch.zeros(state["fills"], case["kv_heads"], page, case["d"], device=DEVICE, dtype=torch.float64), 0
            after = window.clone()
            for b, (m, n) in enumerate(zip(lens, new)):
                old = (m - n) // page * page
                stream = torch.cat([window[wins[b, 0], :, : m - n - old].transpose(0, 1), x[at: at + n].double()])
                for p in range(old // page, m // page):
                    pages[table[b, p]] = stream[p * page - old: (p + 1) * page - old].transpose(0, 1)
                tail = m % page
                fresh = min(tail, n)
                after[wins[b, 1], :, tail - fresh: tail] = x[at + n - fresh: at + n].double().transpose(0, 1)
                at += n
            y = (pages @ forward.T).unflatten(-1, (-1, case["g"]))
            step = (y.abs().amax(-1, keepdim=True) / steps).clamp(min=1e-300)
            out += [((torch.round(y / step) * step).flatten(-2) @ back[s].T).flatten(0, 2), after]
        return out if state["fills"] else out[1::2]
    if sum(n * (m + 1) for m, n in zip(lens, new)) * case["kv_heads"] * case["group"] > 2e9:
        return None
    out, at = [], 0
    for b, (m, n) in enumerate(zip(lens, new)):
        ids = torch.tensor(table[b, : m // page], device=DEVICE, dtype=torch.long)
        k, v = (torch.cat([(_decoded(state[s]["codes"][ids], state[s]["scales"][ids], bits) @ back[s].T).transpose(0, 1).flatten(1, 2),
                           state[s]["window"][wins[b, 1], :, : m % page].double()], 1) for s in "kv")
        here = []
        for h in range(case["kv_heads"]):
            q = state["q"][at: at + n, h * case["group"]: (h + 1) * case["group"]].double()
            a = torch.einsum("igd,td->igt", q, k[h]) * state["scale"]
            late = torch.arange(m, device=DEVICE)[None, :] > torch.arange(m - n, m, device=DEVICE)[:, None]
            a.masked_fill_(late[:, None], -math.inf)
            here.append(torch.softmax(a, -1) @ v[h])
        out.append(torch.cat(here, 1))
        at += n
    return torch.cat(out)
