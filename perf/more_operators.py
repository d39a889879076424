"""More operators of a serving step over a paged cache, and of its training: what is timed of them, in elementary torch and through the library.

  norm      RMS norm of every head of queries and keys with their rotary positions, in one call: ``srft_norm_rotary``
  grad      its gradients, of the inputs and of the norms' weights: ``srft_norm_rotary_backward``
  sliding   causal attention over the pages, of the last ``recent`` tokens and the first ``sinks``: ``srft_pool_attention_sliding``
  shared    causal attention of sequences that have their first pages in common: ``srft_pool_attention_shared``

The cache of one layer is a pool of pages for K and one for V.  A page holds ``page`` tokens of ``kv_heads`` heads as the
quantizer's record (codes, fp32 scales); a sequence's last ``len % page`` tokens are exact fp16 in a window.  A record is
``code * scale`` in the packed transform domain: x = S Q^T diag(1 / lambda) (code * scale), with Q the real packing of the
unitary DFT and S a diagonal of signs.

Sequence b of a call has the query rows ``starts[b] .. starts[b + 1]`` and holds ``lengths[b]`` tokens, these among them; its token j lies
in page ``table[b][j / page]``, or in the window ``windows[b][1]`` if it is behind the last full page.  The sequences
``groups[g] .. groups[g + 1]`` have the pages of their first ``shared[g]`` tokens in common.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------------- cases
def listed() -> list[dict]:
    norm = dict(d=128, rot=128, layout="half", x="f16", y="f16", w="f16", far=32768, stretch=1.0)
    page = dict(d=128, g=32, bits=4, page=16, q="f16")
    slide, share = dict(page, op="sliding"), dict(page, op="shared")
    return [
        # a decode step of 8 sequences, 12 query heads and 2 key heads: all latency
        dict(norm, op="norm", name="norm_step", tokens=8, q_heads=12, kv_heads=2),
        # a prompt of 8192 tokens in bf16, 32 + 8 heads, keys and queries to fp16, positions stretched for a long context
        dict(norm, op="norm", name="norm_prompt", tokens=8192, q_heads=32, kv_heads=8, x="bf16", w="bf16", far=131072, stretch=8.0),
        # the backward pass of a training batch in bf16, 32 + 8 heads
        dict(norm, op="grad", name="grad_batch", tokens=8192, q_heads=32, kv_heads=8, x="bf16", y="bf16", w="bf16"),
        # the same of a small model in fp32: interleaved pairs, the first 64 of 96 channels, an odd number of tokens
        dict(norm, op="grad", name="grad_odd", tokens=1777, q_heads=10, kv_heads=5, d=96, rot=64, layout="pairs", x="f32", y="f32", w="f32"),
        # one decode step of 4 short sequences, 6 query heads to a key head, 128 recent tokens and 4 first ones
        dict(slide, name="sliding_short", seqs=4, len_min=60, len_max=1000, new_min=1, new_max=1, kv_heads=2, group=6, recent=128, sinks=4),
        # one decode step of a serving batch: 48 ragged sequences up to 32768 tokens, 64 query and 8 key heads, 4096 recent tokens
        dict(slide, name="sliding_batch", seqs=48, len_min=500, len_max=32768, new_min=1, new_max=1, kv_heads=8, group=8, recent=4096, sinks=64),
        # a chunk of a long prompt behind the tokens that the cache has already, 32 query and 8 key heads
        dict(slide, name="sliding_chunk", seqs=1, len_min=16384, len_max=16384, new_min=2048, new_max=2048, kv_heads=8, group=4, recent=4096, sinks=16),
        # prompts' chunks and decode steps in one batch, d = 256 with 8-bit codes, pages of 64, bf16 queries
        dict(slide, name="sliding_mixed", seqs=8, len_min=700, len_max=4096, new_min=1, new_max=500, kv_heads=4, group=2, d=256, bits=8, page=64,
             q="bf16", recent=1000, sinks=5),
        # 6 samples of one short prompt, a decode step, 6 query heads to a key head
        dict(share, name="shared_short", groups=1, seqs=6, prefix_min=800, prefix_max=800, own_min=1, own_max=90, new_min=1, new_max=1, kv_heads=2, group=6),
        # a decode step of 64 conversations that begin with the same 16384 tokens, 64 query and 8 key heads
        dict(share, name="shared_batch", groups=1, seqs=64, prefix_min=16384, prefix_max=16384, own_min=20, own_max=1500, new_min=1, new_max=1,
             kv_heads=8, group=8),
        # questions of 40 to 300 tokens about one document of 12000, 32 query and 8 key heads
        dict(share, name="shared_questions", groups=1, seqs=8, prefix_min=12000, prefix_max=12000, own_min=40, own_max=300, new_min=40, new_max=300,
             kv_heads=8, group=4),
        # 5 prompts of 700 to 5000 tokens with 2 to 11 samples each, a decode step, d = 256 with 8-bit codes, pages of 64, bf16 queries
        dict(share, name="shared_groups", groups=5, seqs=31, prefix_min=700, prefix_max=5000, own_min=10, own_max=700, new_min=1, new_max=1, kv_heads=4,
             group=4, d=256, bits=8, page=64, q="bf16"),
    ]


def _log_int(rng: random.Random, lo: float, hi: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random) -> dict:
    op = rng.choice(["norm", "grad", "sliding", "sliding", "shared", "shared"])
    kv = rng.choice([1, 2, 3, 4, 8])
    if op in ("norm", "grad"):
        d = rng.choice([64, 96, 128, 192, 256])
        x = rng.choice(["f16", "bf16", "f32"])
        return dict(op=op, tokens=_log_int(rng, 1, 4096 if x == "f32" or d > 128 else 8192), q_heads=kv * rng.choice([1, 3, 4]), kv_heads=kv, d=d,
                    rot=rng.choice([d, d // 2, 32]), layout=rng.choice(["half", "pairs"]), x=x, y=rng.choice([x, "f16"]) if op == "norm" else x,
                    w=rng.choice([x, "f32"]), far=_log_int(rng, 2048, 1000000), stretch=rng.choice([1.0, 1.0, 4.0, 32.0]))
    d = rng.choice([64, 96, 128, 128, 128, 192, 256])
    page = rng.choice([16, 32, 64, 128])
    if kv % 2 and page == 16:
        page = 32
    shape = dict(op=op, d=d, g=rng.choice([32, 32, 32, 16, d]), bits=rng.choice([4, 4, 8]), page=page, q=rng.choice(["f16", "bf16"]), kv_heads=kv,
                 group=rng.choice([1, 2, 4, 6, 8]))
    if op == "shared":
        new = rng.choice([1, 1, 1, 4, _log_int(rng, 2, 200)])
        groups, prefix, extra = rng.choice([1, 1, 2, 4]), _log_int(rng, 20, 9000), _log_int(rng, 4, 1200)
        return dict(shape, groups=groups, seqs=groups * _log_int(rng, 1, 12) + rng.randrange(3), prefix_min=prefix // rng.choice([1, 1, 3]), prefix_max=prefix,
                    own_min=max(1, new // 2), own_max=new + extra, new_min=max(1, new // 2), new_max=new)
    reach = dict(recent=_log_int(rng, 1, 6000), sinks=rng.choice([0, 0, 1, 4, 16, rng.randrange(1, 300)]))
    kind = rng.choice(["decode", "decode", "chunk", "mixed"])
    if kind == "decode":
        seqs, top, new = _log_int(rng, 1, 48), _log_int(rng, 50, 16000), rng.choice([1, 1, 1, 4])
        return dict(shape, **reach, seqs=seqs, len_min=max(1, int(top * rng.uniform(0.02, 1.0))), len_max=top, new_min=1, new_max=new)
    seqs = rng.randint(1, 3) if kind == "chunk" else rng.randint(3, 8)
    new = _log_int(rng, 20, 800)
    top = new + _log_int(rng, 1, 5000)
    return dict(shape, **reach, seqs=seqs, len_min=max(1, top // rng.choice([1, 2, 8])), len_max=top, new_min=new if kind == "chunk" else 1, new_max=new)


def _spread(n: int, low: int, high: int, power: int) -> np.ndarray:
    """n whole numbers from low to high, in no order, odd ones among them; the first is the largest."""
    at = (np.arange(n) * 7 % n + 0.5) / n if n % 7 else (np.arange(n) + 0.5) / n
    at[0] = 1.0
    return np.rint(low + (high - low) * at ** power).astype(np.int64)


def _ragged(case: dict) -> dict:
    """A case's sequences: their lengths, their new tokens and, where they share pages, the groups and the tokens of their pages in common."""
    n = case["seqs"]
    new = _spread(n, case["new_min"], case["new_max"], 1 if case["new_min"] * 4 > case["new_max"] else 4)
    if case["op"] == "sliding":
        lens = _spread(n, case["len_min"], case["len_max"], 2)
        return {"lens": lens, "new": np.minimum(new, lens), "common": np.zeros(n, np.int64)}
    groups = np.rint(np.linspace(0, 1, case["groups"] + 1) ** 1.5 * n).astype(np.int64)
    prefix = _spread(case["groups"], case["prefix_min"], case["prefix_max"], 1) // case["page"] * case["page"]
    extra = _spread(n, case["own_min"], case["own_max"], 2)
    common = np.repeat(prefix, np.diff(groups))
    return {"lens": common + extra, "new": np.minimum(new, extra), "common": common, "groups": groups, "shared": prefix}


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


def _prepare_norm(case: dict, gen: torch.Generator) -> dict:
    n, hq, hk, d = case["tokens"], case["q_heads"], case["kv_heads"], case["d"]
    heads = hq + 2 * hk
    gain = torch.exp(0.5 * torch.randn(1, heads, 1, device=DEVICE, generator=gen))                   # (heads of several sizes)
    packed = (torch.randn(n, heads, d, device=DEVICE, generator=gen) * gain).to(DTYPES[case["x"]])   # q, k and v next to each other
    st = {"q": packed[:, :hq], "k": packed[:, hq: hq + hk],
          "positions": torch.randint(0, case["far"], (n,), device=DEVICE, generator=gen, dtype=torch.int32),
          "freq": torch.tensor(_frequencies(case), device=DEVICE), "factor": 1.0 + 0.1 * math.log(case["stretch"])}
    for x, h in (("q", hq), ("k", hk)):
        st[x + "_weight"] = (1.0 + 0.3 * torch.randn(d, device=DEVICE, generator=gen)).to(DTYPES[case["w"]])
        st[x + "_out"] = torch.empty(n, h, d, device=DEVICE, dtype=DTYPES[case["y"]])
        if case["op"] == "grad":
            st[x + "_dy"] = torch.randn(n, h, d, device=DEVICE, generator=gen).to(DTYPES[case["y"]])
            st[x + "_dweight"] = torch.empty(d, device=DEVICE)
    if own and case["op"] == "grad":
        from paper_2605_05699_amd import binding as B
        st["workspace"] = torch.empty(B.srft_norm_rotary_backward_workspace_bytes(2, d), device=DEVICE, dtype=torch.uint8)
    return st


def _prepare_pages(case: dict, seed: int, gen: torch.Generator) -> dict:
    d, g, bits, page, heads = (case[k] for k in ("d", "g", "bits", "page", "kv_heads"))
    st = _ragged(case)
    lens, new, common = st["lens"], st["new"], st["common"] // page
    n, full = len(lens), lens // page
    rng = np.random.RandomState(seed % (1 << 32))
    # every page has a place of its own in the pool, in no order; those that a group shares are its first sequence's
    first = np.arange(n) if case["op"] == "sliding" else np.repeat(st["groups"][:-1], np.diff(st["groups"]))
    mine = np.where(np.arange(n) == first, full, full - common)
    pages = max(1, int(mine.sum()))
    order, table = rng.permutation(pages), np.full((n, int(full.max()) + 1), -1, np.int32)
    for b in range(n):
        table[b, full[b] - mine[b]: full[b]], order = order[: mine[b]], order[mine[b]:]
        table[b, : full[b] - mine[b]] = table[first[b], : full[b] - mine[b]]
    slots = rng.permutation(2 * n).reshape(n, 2)[:, :1].repeat(2, 1).astype(np.int32)
    on = lambda a: torch.tensor(np.ascontiguousarray(a).astype(np.int32), device=DEVICE)      # noqa: E731
    st |= {"max_new": int(new.max()), "max_len": int(lens.max()), "table": on(table), "windows": on(slots), "lengths": on(lens),
           "starts": on(np.concatenate([[0], np.cumsum(new)])), "most_common": int(common.max())}
    if case["op"] == "shared":
        st["groups_dev"], st["shared_dev"], st["common_dev"] = on(st["groups"]), on(st["shared"]), on(common)
    for name, plan_seed in zip("kv", (seed * 1_000_003 + 1, seed * 1_000_003 + 2)):
        lam, w, r = _constants(plan_seed, d)
        w32 = torch.tensor(w, device=DEVICE, dtype=torch.float32)
        codes = torch.zeros(pages, heads, page, d * bits // 8, device=DEVICE, dtype=torch.uint8)
        scales = torch.zeros(pages, heads, page, d // g, device=DEVICE)
        for at in range(0, pages, 4096):
            m = min(4096, pages - at)
            codes[at: at + m], scales[at: at + m] = _quantize(_rows(gen, (m, heads, page, d), name == "k"), w32, g, bits)
        st[name] = {"seed": plan_seed, "lam": lam, "r": torch.tensor(r, device=DEVICE, dtype=torch.float32), "codes": codes, "scales": scales,
                    "window": _rows(gen, (2 * n, heads, page, d), name == "k")}
    st["q"] = torch.randn(int(new.sum()), heads * case["group"], d, device=DEVICE, generator=gen).to(DTYPES[case["q"]])
    st["out"] = torch.empty_like(st["q"])
    st["scale"] = d ** -0.5
    return st


def _keep(case: dict, st: dict) -> None:
    """What a program keeps between steps beside its buffers: the handle, the batch's description and a workspace."""
    from paper_2605_05699_amd import binding as B
    plans = [B.Plan(case["d"], case["g"], st[x]["seed"], st[x]["lam"], bits=case["bits"]) for x in "kv"]
    st["pool"] = B.PagePool(*plans, *[(st[x]["codes"], st[x]["scales"], st[x]["window"]) for x in "kv"])
    st["seqs"] = B.PagedSeqs(st["table"], st["windows"], st["lengths"], st["starts"], max_new=st["max_new"], max_length=st["max_len"])
    n, heads = st["q"].shape[:2]
    if case["op"] == "shared":
        st["prefixes"] = B.SharedPrefixes(st["groups_dev"], st["shared_dev"])
        size = B.srft_pool_attention_shared_workspace_bytes(st["pool"], st["seqs"], st["prefixes"], n, heads)
    else:
        size = B.srft_pool_attention_sliding_workspace_bytes(st["pool"], st["seqs"], n, heads)
    st["workspace"] = torch.empty(size, device=DEVICE, dtype=torch.uint8)


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(DEVICE)
    gen.manual_seed(seed)
    if case["op"] in ("norm", "grad"):
        st = _prepare_norm(case, gen)
    else:
        st = _prepare_pages(case, seed, gen)
        if own:
            _keep(case, st)
    st["case"] = case
    return st


# --------------------------------------------------------------------------------------------------- the plain forms, and ours
def _turned(st: dict, x: torch.Tensor, sign: float) -> torch.Tensor:
    case, rot = st["case"], st["case"]["rot"]
    angle = st["positions"].double()[:, None, None] * st["freq"]             # (64 bits: far positions)
    cos, sin = (torch.cos(angle) * st["factor"]).float(), (torch.sin(angle) * (sign * st["factor"])).float()
    part, rest = x[..., :rot], x[..., rot:]
    a, b = (part[..., : rot // 2], part[..., rot // 2:]) if case["layout"] == "half" else (part[..., 0::2], part[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.cat([torch.cat([u, v], -1) if case["layout"] == "half" else torch.stack([u, v], -1).flatten(-2), rest], -1)


def _plain_norm(st: dict, name: str) -> torch.Tensor:
    x = st[name].float()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    return _turned(st, x * r * st[name + "_weight"].float(), 1.0).to(DTYPES[st["case"]["y"]])


def _plain_grad(st: dict, name: str) -> list[torch.Tensor]:
    x = st[name].float()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    h, g = x * r, _turned(st, st[name + "_dy"].float(), -1.0)
    dn = g * st[name + "_weight"].float()
    dx = r * (dn - h * (dn * h).mean(-1, keepdim=True))
    return [dx.to(st[name].dtype), (g * h).double().sum((0, 1)).float()]


def _pages_of(st: dict, name: str, table: torch.Tensor) -> torch.Tensor:
    """The stored tokens of pages [n, m] -> fp32 [n, head, m * page, d]."""
    s, at = st[name], table.clamp(min=0).long()
    return (_values(s["codes"][at], s["scales"][at], st["case"]["bits"]) @ s["r"].T).transpose(1, 2).flatten(2, 3)


def _scores(st: dict, q: torch.Tensor, k: torch.Tensor, see: torch.Tensor) -> torch.Tensor:
    """q [n, head, rows, d], k [n, head, tokens, d], see [n, rows, tokens]."""
    return torch.where(see[:, None], torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"], -math.inf)


def _plain_attention(st: dict) -> torch.Tensor:
    case = st["case"]
    page, heads, group = case["page"], case["kv_heads"], case["group"]
    lengths, starts, far = st["lengths"].long(), st["starts"].long(), 1 << 40
    shared = case["op"] == "shared"
    common = st["common_dev"].long() if shared else torch.zeros_like(lengths)                # pages in front of a sequence's own
    most = (st["lens"] // page - st["common"] // page).max()
    column = common[:, None] + torch.arange(max(1, int(most)), device=DEVICE)[None]
    table = st["table"].gather(1, column.clamp(max=st["table"].shape[1] - 1))
    full = lengths // page * page
    j = (column[:, :, None] * page + torch.arange(page, device=DEVICE)).flatten(1)
    behind = full[:, None] + torch.arange(page, device=DEVICE)[None]
    pos = torch.cat([torch.where(j < full[:, None], j, far), torch.where(behind < lengths[:, None], behind, far)], 1)
    k, v = (torch.cat([_pages_of(st, x, table), st[x]["window"][st["windows"][:, 1].long()].float()], 2) for x in "kv")
    new = starts[1:] - starts[:-1]
    i = torch.arange(st["max_new"], device=DEVICE)[None]
    row = (starts[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)
    limit = torch.where(i < new[:, None], (lengths - new)[:, None] + i, -1).repeat_interleave(group, 1)[:, :, None]
    heads_of = lambda x: x.unflatten(2, (heads, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # noqa: E731  [n, head, token * group, d]
    see = pos[:, None, :] <= limit
    if not shared:
        see &= (pos[:, None, :] > limit - case["recent"]) | (pos[:, None, :] < case["sinks"])
    q = st["q"].float()
    s = _scores(st, heads_of(q[row]), k, see)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
    total, o = p.sum(-1, keepdim=True), torch.matmul(p, v)
    r = torch.arange(q.shape[0], device=DEVICE)
    seq = torch.searchsorted(starts, r, right=True) - 1
    rows_of = lambda x, a, b: x.unflatten(2, (-1, group)).transpose(1, 2)[a, b]               # noqa: E731  [new tokens, head, group, ..]
    o, total, top = (rows_of(x, seq, r - starts[seq]) for x in (o, total, top))
    if shared and st["most_common"] > 0:                     # the pages in common, once for all rows of a group
        groups = st["groups_dev"].long()
        at = starts[groups]
        i = torch.arange(int(np.add.reduceat(st["new"], st["groups"][:-1]).max()), device=DEVICE)[None]
        first = st["table"][groups[:-1].clamp(max=len(lengths) - 1), : st["most_common"]]
        token = torch.arange(st["most_common"] * page, device=DEVICE)[None, None]
        see = (token < st["shared_dev"].long()[:, None, None]).expand(-1, i.shape[1] * group, -1)
        s = _scores(st, heads_of(q[(at[:-1, None] + i).clamp(max=q.shape[0] - 1)]), _pages_of(st, "k", first), see)
        g = torch.searchsorted(at, r, right=True) - 1
        far_top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(far_top > -math.inf, far_top, 0.0))
        far_o, far_total, far_top = (rows_of(x, g, r - at[g]) for x in (torch.matmul(p, _pages_of(st, "v", first)), p.sum(-1, keepdim=True), far_top))
        both = torch.maximum(top, far_top)
        a, b = torch.exp(top - both), torch.exp(far_top - both)
        o, total = o * a + far_o * b, total * a + far_total * b
    return (o / torch.where(total > 0, total, 1.0)).flatten(1, 2).to(st["q"].dtype)


def run(state: dict):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2605_05699_amd import binding as B
        if op == "norm":
            B.srft_norm_rotary([(state[x], state[x + "_weight"], state[x + "_out"]) for x in "qk"], state["positions"], state["freq"], EPS,
                               layout=case["layout"], factor=state["factor"])
            return [state["q_out"], state["k_out"]]
        if op == "grad":
            # dx goes to a packed gradient of q and k in a program; here each has a tensor of its own
            B.srft_norm_rotary_backward([(state[x + "_dy"], state[x], state[x + "_weight"], state[x + "_out"], state[x + "_dweight"]) for x in "qk"],
                                        state["positions"], state["freq"], EPS, state["workspace"], layout=case["layout"], factor=state["factor"])
            return [state[x + y] for x in "qk" for y in ("_out", "_dweight")]
        if op == "sliding":
            B.srft_pool_attention_sliding(state["pool"], state["seqs"], state["q"], state["scale"], case["recent"], case["sinks"], state["out"],
                                          state["workspace"])
        else:
            B.srft_pool_attention_shared(state["pool"], state["seqs"], state["prefixes"], state["q"], state["scale"], state["out"], state["workspace"])
        return state["out"]
    if op == "norm":
        return [_plain_norm(state, x) for x in "qk"]
    if op == "grad":
        return [y for x in "qk" for y in _plain_grad(state, x)]
    return _plain_attention(state)


# ------------------------------------------------------------------------------------------------------------------- the work
def work(case: dict) -> dict:
    d = case["d"]
    size = {"f16": 2, "bf16": 2, "f32": 4}
    if case["op"] in ("norm", "grad"):
        n, x, y = case["tokens"] * (case["q_heads"] + case["kv_heads"]), size[case["x"]], size[case["y"]]
        if case["op"] == "norm":
            return {"bytes": n * d * (x + y) + 4 * case["tokens"] + 2 * d * size[case["w"]] + 4 * case["rot"], "flops": n * (4 * d + 3 * case["rot"])}
        return {"bytes": n * d * (2 * x + y) + 4 * case["tokens"] + 2 * d * (size[case["w"]] + 4) + 4 * case["rot"], "flops": n * (11 * d + 3 * case["rot"])}
    heads, page = case["kv_heads"], case["page"]
    record = d * case["bits"] // 8 + 4 * (d // case["g"])
    st = _ragged(case)
    rows, held, tail, pairs = heads * case["group"] * int(st["new"].sum()), 0, 0, 0
    for m, n, c in zip(st["lens"].tolist(), st["new"].tolist(), st["common"].tolist()):
        if case["op"] == "sliding":
            last = np.arange(m - n, m)
            first = np.maximum(last - case["recent"] + 1, 0)
            sinks = np.minimum(case["sinks"], first)
            pairs += int((last + 1 - first + sinks).sum())
            full, seen = m // page * page, np.r_[0: int(sinks[0]), int(first[0]): m]         # (tokens that any row sees)
            held, tail = held + int((seen < full).sum()), tail + int((seen >= full).sum())
        else:
            pairs += n * (m - n) + n * (n + 1) // 2
            held, tail = held + m // page * page - c, tail + m % page
    if case["op"] == "shared":
        held += int(st["shared"].sum())
    return {"bytes": 2 * heads * (held * record + tail * 2 * d) + 2 * rows * 2 * d, "flops": 4 * pairs * heads * case["group"] * d}


# --------------------------------------------------------------------------------------------------- by definition, in 64 bits
def _decoded(codes: torch.Tensor, scales: torch.Tensor, bits: int) -> torch.Tensor:
    """Stored rows in 64 bits: what each byte stands for is looked up."""
    low = [(i & 15) - 16 * (i >> 3 & 1) for i in range(256)]
    pair = [(a, low[i >> 4]) for i, a in enumerate(low)] if bits == 4 else [(i - 256 * (i >> 7),) for i in range(256)]
    q = torch.tensor(pair, device=DEVICE, dtype=torch.float64)[codes.long()].flatten(-2)
    return q * scales.double().repeat_interleave(q.shape[-1] // scales.shape[-1], -1)


def _exact_norm(case: dict, st: dict):
    f = torch.tensor(_frequencies(case), device=DEVICE)
    z = torch.polar(torch.full((case["tokens"], len(f)), 1.0 + 0.1 * math.log(case["stretch"]), device=DEVICE, dtype=torch.float64),
                    st["positions"].double()[:, None] * f)[:, None]
    r = case["rot"]
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))

    def turn(y, by):
        y = y.clone()
        t = torch.complex(y[..., first], y[..., second]) * by
        y[..., first], y[..., second] = t.real, t.imag
        return y
    out = []
    for name in "qk":
        x, w = st[name].double(), st[name + "_weight"].double()
        size = (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / case["d"] + EPS) ** 0.5
        if case["op"] == "norm":
            out.append(turn(x / size * w, z))
            continue
        # y = turn(w x / size): its derivative along x is w / size - w x (x / d) / size^3
        g = turn(st[name + "_dy"].double(), z.conj())
        out += [g * w / size - x * ((g * w * x).sum(-1, keepdim=True) / (case["d"] * size ** 3)), (g * x / size).flatten(0, 1).sum(0)]
    return out


def exact(case: dict, seed: int):
    state = prepare(case, seed)
    if case["op"] in ("norm", "grad"):
        return _exact_norm(case, state)
    lens, new = state["lens"].tolist(), state["new"].tolist()
    table, wins, page, bits = state["table"].cpu().numpy(), state["windows"].cpu().numpy(), case["page"], case["bits"]
    back = {s: torch.tensor(_constants(state[s]["seed"], case["d"])[2], device=DEVICE) for s in "kv"}
    if sum(n * (m + 1) for m, n in zip(lens, new)) * case["kv_heads"] * case["group"] > 2e9:
        return None
    out, at = [], 0
    for b, (m, n) in enumerate(zip(lens, new)):
        ids = torch.tensor(table[b, : m // page], device=DEVICE, dtype=torch.long)
        k, v = (torch.cat([(_decoded(state[s]["codes"][ids], state[s]["scales"][ids], bits) @ back[s].T).transpose(0, 1).flatten(1, 2),
                           state[s]["window"][wins[b, 1], :, : m % page].double()], 1) for s in "kv")
        token, mine = torch.arange(m, device=DEVICE)[None, :], torch.arange(m - n, m, device=DEVICE)[:, None]
        hidden = token > mine
        if case["op"] == "sliding":
            hidden |= (mine - token >= case["recent"]) & (token >= case["sinks"])
        here = []
        for h in range(case["kv_heads"]):
            q = state["q"][at: at + n, h * case["group"]: (h + 1) * case["group"]].double()
            a = torch.einsum("igd,td->igt", q, k[h]) * state["scale"]
            a.masked_fill_(hidden[:, None], -math.inf)
            here.append(torch.softmax(a, -1) @ v[h])
        out.append(torch.cat(here, 1))
        at += n
    return torch.cat(out)
