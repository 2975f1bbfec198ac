"""The operators of a paged KV cache, as cases that can be timed and checked.

The prompt of a sequence may be clustered; the tokens that are decoded after it, and layers that stay dense, live in a
paged cache: a pool of pages of ``page`` tokens each, and per sequence a table of the pages that hold its tokens.

* ``append``  new keys and values go to their places in the pages, rotated to their positions on the way, and the
              queries of the same tokens are rotated with them (``dp_append_kv``)
* ``paged``   one query token per sequence attends to the rows of its pages, all of them or those from a first row on;
              where a ``prior`` is given, the attention over the rest of the context (its output and log-normaliser, as
              a step over the clustered prompt leaves them) is joined (``dp_paged_decode``)
* ``shared``  the same for a batch in which groups of sequences share their first rows (a system prompt, a document
              that many requests ask about): the shared rows are read once for a whole group
              (``dp_shared_prefix_decode``)

head_dim 128, bf16 pages, as everywhere in this repository; lengths from one token to 131072, batches up to 64, groups
of 1 to 8 query heads per KV head, pages of 1 to 256 tokens, both orders of heads and tokens inside a page.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DIM = 128
ROW = 2 * DIM  # bytes of one bf16 row

APPEND = dict(kind="append", seqs=1, kv_heads=8, group=4, tokens=1, ragged=False, context=4096, page=16, layout="head",
              input="bf16", rotated=128, pairs="halves")
PAGED = dict(kind="paged", seqs=1, kv_heads=8, group=4, context=4096, ragged=False, idle=0, first=False, prior=False,
             page=16, layout="head", out="bf16")
SHARED = dict(kind="shared", seqs=8, groups=1, kv_heads=8, group=4, prefix=2048, context=256, ragged=True, idle=0,
              page=16, layout="head", out="bf16")


def listed():
    return [
        # one sequence decodes one token: what a call costs when there is next to nothing to move
        dict(APPEND, name="append_one"),
        # a decode step of a full batch, every sequence at another length
        dict(APPEND, name="append_batch64", seqs=64, ragged=True, context=1024),
        # a few prompts of odd lengths join the batch; projections in fp32, half of each head rotated, pairs side by
        # side, pages with the tokens outside and the heads inside
        dict(APPEND, name="append_prompts", seqs=5, tokens=5003, ragged=True, context=6000, page=64, layout="token",
             input="f32", rotated=64, pairs="adjacent"),
        # one long prompt
        dict(APPEND, name="append_128k", tokens=131072, context=131072, page=64),
        # one short sequence, one KV head
        dict(PAGED, name="paged_short", kv_heads=1, context=1000, out="f32"),
        # the tokens decoded after clustered prompts, joined with the attention over those
        dict(PAGED, name="paged_tail", seqs=32, context=700, ragged=True, first=True, prior=True, out="f32"),
        # continuous batching of a dense layer: sequences of different lengths, two slots of the batch idle
        dict(PAGED, name="paged_batch16", seqs=16, context=65536, ragged=True, idle=2),
        # one long sequence
        dict(PAGED, name="paged_128k", context=131072, page=64),
        # four long sequences, wide groups, large pages with the tokens outside: the largest read
        dict(PAGED, name="paged_gqa8_128k", seqs=4, group=8, context=131072, page=256, layout="token", out="f32"),
        # a few requests behind a short system prompt
        dict(SHARED, name="shared_2k"),
        # many requests about one long document
        dict(SHARED, name="shared_64x32k", seqs=64, prefix=32768, context=1024, page=64),
        # several documents with groups of odd sizes, odd lengths, idle slots, wide groups of heads
        dict(SHARED, name="shared_groups", seqs=37, groups=3, kv_heads=4, group=8, prefix=20011, context=777, idle=3,
             out="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "paged", "shared"])
    common = dict(kv_heads=rng.choice([1, 2, 4, 8, 8]), group=rng.choice([1, 2, 4, 4, 5, 7, 8]),
                  page=rng.choice([1, 8, 16, 16, 32, 64, 256]), layout=rng.choice(["head", "head", "token"]))
    while True:
        if kind == "append":
            case = dict(APPEND, **common)
            case.update(seqs=_log_int(rng, 1, 64), tokens=rng.choice([1, 1, 2, _log_int(rng, 3, 131072)]),
                        ragged=rng.random() < 0.6, input=rng.choice(["bf16", "bf16", "f32"]),
                        rotated=rng.choice([128, 128, 64, 32, 0]), pairs=rng.choice(["halves", "adjacent"]))
            case["context"] = case["tokens"] + _log_int(rng, 1, 4096)
            if case["seqs"] * case["context"] * case["kv_heads"] > 8 * 131072:
                continue
            if case["seqs"] * case["tokens"] * case["kv_heads"] * case["group"] > 32 * 131072:
                continue
            if case["input"] == "f32" and case["seqs"] * case["tokens"] * case["kv_heads"] * case["group"] > 16 * 131072:
                continue
            return case
        out = rng.choice(["bf16", "f32"])
        if kind == "paged":
            case = dict(PAGED, **common)
            case.update(seqs=_log_int(rng, 1, 64), context=_log_int(rng, 1, 131072), ragged=rng.random() < 0.6,
                        first=rng.random() < 0.3, prior=rng.random() < 0.4, out=out)
            if case["seqs"] > 2 and rng.random() < 0.3:
                case["idle"] = rng.randint(1, case["seqs"] // 2)
            if case["seqs"] * case["context"] * case["kv_heads"] > 4 * 8 * 131072:
                continue
            return case
        case = dict(SHARED, **common)
        case.update(seqs=_log_int(rng, 2, 64), groups=rng.choice([1, 1, 2, 4]), prefix=_log_int(rng, 16, 131072),
                    context=_log_int(rng, 1, 4096), ragged=rng.random() < 0.7, out=out)
        case["groups"] = min(case["groups"], case["seqs"])
        if case["seqs"] > 4 and rng.random() < 0.3:
            case["idle"] = rng.randint(1, case["seqs"] // 3)
        heads = case["kv_heads"] * case["group"]
        if case["seqs"] * heads * (case["prefix"] + case["context"]) > 64 * 32 * 33792:
            continue
        if (case["groups"] * case["prefix"] + case["seqs"] * case["context"]) * case["kv_heads"] > 8 * 131072:
            continue
        return case


def _spread(i, top):
    """The i-th of a ragged series of lengths of at most ``top``, from about a quarter of it upwards."""
    return max(1, int(top * (0.25 + 0.75 * ((i + 1) * 0.6180339887 % 1.0))))


def _idle(case):
    """The idle slots of the batch, spread over it."""
    n = case.get("idle", 0)
    return {(2 * i + 1) * case["seqs"] // (2 * n) for i in range(n)}


def _new(case):
    """New tokens of each sequence of an append."""
    return [_spread(i, case["tokens"]) if case["ragged"] else case["tokens"] for i in range(case["seqs"])]


def _groups(case):
    """First sequence of each group of a shared batch, and the end: uneven groups where there are several."""
    n, more = case["groups"], case["seqs"] - case["groups"]
    return [i + more * i * i // (n * n) for i in range(n + 1)]


def _shared(case):
    """Shared rows of each group."""
    return [case["prefix"]] + [_spread(i, case["prefix"]) for i in range(case["groups"] - 1)]


def _lens(case):
    """Rows of each sequence in the cache, its new tokens and its shared rows among them."""
    tops = [_spread(i, case["context"]) if case["ragged"] else case["context"] for i in range(case["seqs"])]
    tops[0] = case["context"]
    if case["kind"] == "append":
        return [max(a, b) for a, b in zip(tops, _new(case))]
    if case["kind"] == "shared":
        tops = [n + m for n, m in zip(tops, _per_seq(case))]
    idle = _idle(case)
    return [0 if s in idle else n for s, n in enumerate(tops)]


def _first(case):
    """First attended row of each sequence: the rows before it are elsewhere."""
    return [n * (s % 3) // 4 for s, n in enumerate(_lens(case))]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    kvh, heads, seqs, page = case["kv_heads"], case["kv_heads"] * case["group"], case["seqs"], case["page"]
    lens = _lens(case)
    need = [(n + page - 1) // page for n in lens]
    width, pool = max(max(need), 1), sum(need) + 7

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    # the tables of a pool that was in use before: pages in no order, -1 where a sequence has none
    place = torch.arange(width, device="cuda")
    need, start = ints(need)[:, None], ints([sum(need[:s]) for s in range(seqs)])[:, None]
    order = torch.randperm(pool, generator=gen, device="cuda", dtype=torch.int32)
    table = torch.where(place < need, order[(start + place).clamp(max=pool - 1)], -1)
    shape = (pool, page, kvh, DIM) if case["layout"] == "token" else (pool, kvh, page, DIM)
    k, v = normal(*shape, dtype=torch.bfloat16), normal(*shape, dtype=torch.bfloat16)
    if case["kind"] == "shared":
        cuts = _groups(case)
        for g, rows in enumerate(_shared(case)):
            users = [s for s in range(cuts[g], cuts[g + 1]) if lens[s]]
            for s in users[1:]:
                # pages that lie wholly inside the shared rows are the same; the one in which those end is a copy
                if rows % page:
                    old, new = table[users[0], rows // page].long(), table[s, rows // page].long()
                    k[new], v[new] = k[old], v[old]
                table[s, :rows // page] = table[users[0], :rows // page]
    if case["layout"] == "token":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    state = {"kind": case["kind"], "group": case["group"], "k": k, "v": v, "table": table, "lens": ints(lens),
             "longest": max(max(lens), 1), "keep": {}}
    if case["kind"] == "append":
        new = _new(case)
        n = sum(new)
        # queries, keys and values side by side, as one projection leaves them
        x = normal(n, heads + 2 * kvh, DIM, dtype=torch.float32 if case["input"] == "f32" else torch.bfloat16)
        ptr = [0]
        for m in new:
            ptr.append(ptr[-1] + m)
        rot = case["rotated"]
        state.update(q_new=x[:, :heads], k_new=x[:, heads:heads + kvh], v_new=x[:, heads + kvh:],
                     # (one new token per sequence needs no list of where a sequence's tokens begin)
                     ptr=None if case["tokens"] == 1 else ints(ptr),
                     freq=500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float32) / max(rot, 1)),
                     adjacent=case["pairs"] == "adjacent",
                     q_out=torch.empty(n, heads, DIM, device="cuda", dtype=torch.bfloat16))
        return state
    # queries from flat to peaked heads
    sharp = torch.tensor([rng.uniform(0.3, 3.0) for _ in range(heads)], device="cuda")
    state["q"] = (normal(seqs, heads, DIM) * sharp[:, None]).to(torch.bfloat16)
    state["out"] = torch.empty(seqs, heads, DIM, device="cuda",
                               dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16)
    state["lse"] = torch.empty(seqs, heads, device="cuda")
    if case["kind"] == "shared":
        cuts = _groups(case)
        state.update(group_ptr=ints(cuts), shared=ints(_shared(case)), longest_shared=max(_shared(case)),
                     longest_own=max(1, max(n - m if n >= m else n for n, m in zip(lens, _per_seq(case)))),
                     most=max(b - a for a, b in zip(cuts, cuts[1:])))
        return state
    state["first"] = ints(_first(case)) if case["first"] else None
    state["prior"] = None
    if case["prior"]:
        state["prior"] = 0.1 * normal(seqs, heads, DIM), 7.0 + normal(seqs, heads)
    return state


def _per_seq(case):
    """Shared rows of each sequence's group."""
    cuts, rows = _groups(case), _shared(case)
    return [rows[g] for g in range(case["groups"]) for _ in range(cuts[g], cuts[g + 1])]


def run(state):
    if own:
        return _own(state)
    return {"append": _append, "paged": _paged, "shared": _shared_prefix}[state["kind"]](state)


def _own(state):
    import paper_2602_05191_amd as dp

    keep, kind = state["keep"], state["kind"]
    if not keep:  # what a serving loop keeps from step to step: the handle of its cache, a workspace, the bound call
        if kind == "append":
            cache = dp.PagedCache(state["k"], state["v"], state["table"], state["lens"], state["longest"], state["q_new"].shape[1])
            keep["call"] = dp.BoundCall(dp.dp_append_kv, cache, state["k_new"], state["v_new"], state["freq"], q=state["q_new"],
                                        q_out=state["q_out"], tok_ptr=state["ptr"], adjacent_pairs=state["adjacent"])
            keep["result"] = state["q_out"], state["k"], state["v"]
        else:
            cache = dp.PagedCache(state["k"], state["v"], state["table"], state["lens"], state["longest"], state["q"].shape[1])
            keep["result"] = state["out"], state["lse"]
        if kind == "paged":
            workspace = torch.empty(dp.dp_paged_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
            prior_out, prior_lse = state["prior"] or (None, None)
            keep["call"] = dp.BoundCall(dp.dp_paged_decode, cache, state["q"], state["out"], state["lse"], workspace,
                                        first_rows=state["first"], prior_out=prior_out, prior_lse=prior_lse)
        if kind == "shared":
            prefix = dp.SharedPrefix(state["group_ptr"], state["shared"], state["most"], state["longest_shared"])
            workspace = torch.empty(dp.dp_shared_prefix_workspace_bytes(cache, prefix), dtype=torch.uint8, device="cuda")
            keep["call"] = dp.BoundCall(dp.dp_shared_prefix_decode, cache, prefix, state["q"], state["out"], state["lse"], workspace)
    keep["call"]()
    return keep["result"]


# ---------------------------------------------------------------- plain forms --
def _rotate(x, cos, sin, adjacent):
    """The first 2 x cos.shape[-1] dimensions of x [n, heads, DIM] turned by pairs, in fp32."""
    x = x.float()
    half = cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    turned, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if adjacent else (turned[..., :half], turned[..., half:])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((a, b), -1).flatten(-2) if adjacent else torch.cat((a, b), -1)
    return torch.cat((turned, rest), -1).to(torch.bfloat16)


def _append(state):
    n, page = state["k_new"].shape[0], state["k"].shape[2]
    token = torch.arange(n, device="cuda")
    ptr = torch.arange(n + 1, device="cuda") if state["ptr"] is None else state["ptr"].long()
    seq = torch.searchsorted(ptr, token, right=True) - 1
    at = state["lens"].long()[seq] - (ptr[seq + 1] - token)  # the new tokens are the last of their sequence
    angle = at.double()[:, None] * state["freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    where, slot = state["table"].long()[seq, at // page], at % page
    state["k"][where, :, slot] = _rotate(state["k_new"], cos, sin, state["adjacent"])
    state["v"][where, :, slot] = state["v_new"].to(torch.bfloat16)
    return _rotate(state["q_new"], cos, sin, state["adjacent"]), state["k"], state["v"]


def _rows(pages, table, first, count):
    """Rows first[i] .. first[i] + count - 1 of every line of a page table: fp32 [lines, kv_heads, count, DIM]. Places
    outside the table give some row; the caller masks them."""
    page = pages.shape[2]
    at = first.long()[:, None] + torch.arange(count, device="cuda")
    where = table.long().gather(1, (at // page).clamp(max=table.shape[1] - 1)).clamp(min=0)
    return pages[where, :, at % page].transpose(1, 2).float()


def _softmax(x):
    """exp(x - max), the sum, the max, over the last dimension; a line of nothing but -inf gives zeros."""
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - top.clamp(min=torch.finfo(torch.float32).min))
    return p, p.sum(-1, keepdim=True), top


def _finish(state, o, total, top):
    """o / total (zero where there is nothing) and the log-normaliser, in the caller's layout."""
    out = torch.where(total > 0, o / total, torch.zeros_like(o))
    return out.flatten(1, 2).to(state["out"].dtype), (top + total.log()).flatten(1)


def _paged(state):
    q, kvh = state["q"].float(), state["k"].shape[1]
    seqs, heads = q.shape[:2]
    count, first = state["longest"], torch.zeros_like(state["lens"])
    if state["first"] is not None:
        first = state["first"]
    k = _rows(state["k"], state["table"], first, count)
    x = torch.matmul(q.view(seqs, kvh, heads // kvh, DIM) / math.sqrt(DIM), k.transpose(2, 3))
    del k
    live = torch.arange(count, device="cuda") < (state["lens"] - first)[:, None]
    p, total, top = _softmax(x.masked_fill(~live[:, None, None], -math.inf))
    v = _rows(state["v"], state["table"], first, count)
    o = torch.matmul(p, v)
    if state["prior"]:
        prior_out, prior_lse = state["prior"]
        old = prior_lse.view_as(top)
        both = torch.maximum(top, old)
        here, there = torch.exp(top - both), torch.exp(old - both)
        o, total, top = o * here + prior_out.view_as(o) * there, total * here + there, both
    return _finish(state, o, total, top)


def _shared_prefix(state):
    q, kvh = state["q"].float() / math.sqrt(DIM), state["k"].shape[1]
    seqs, heads = q.shape[:2]
    group, most = heads // kvh, state["most"]
    ptr, lens = state["group_ptr"].long(), state["lens"].long()
    groups, seq = ptr.shape[0] - 1, torch.arange(seqs, device="cuda")
    mine = torch.searchsorted(ptr, seq, right=True) - 1
    place = seq - ptr[mine]
    q = q.view(seqs, kvh, group, DIM)
    # the shared rows, once per group: the queries of its sequences side by side
    stacked = q.new_zeros(groups, most, kvh, group, DIM)
    stacked[mine, place] = q
    stacked = stacked.transpose(1, 2).flatten(2, 3)
    n = state["shared"].long()[mine]
    n = torch.where(lens >= n, n, torch.zeros_like(n))  # a shorter sequence (an idle slot) shares nothing
    # (read through the table of the group's first sequence that has them)
    reader = torch.full_like(ptr[:-1], seqs - 1).scatter_reduce(0, mine, torch.where(n > 0, seq, seqs - 1), "amin")
    table, zero = state["table"][reader], torch.zeros_like(reader)
    x = torch.matmul(stacked, _rows(state["k"], table, zero, state["longest_shared"]).transpose(2, 3))
    x = x.view(groups, kvh, most, group, -1).transpose(1, 2)[mine, place]
    live = torch.arange(state["longest_shared"], device="cuda") < n[:, None]
    x = x.masked_fill(~live[:, None, None], -math.inf)
    # every sequence's own rows
    count = state["longest_own"]
    y = torch.matmul(q, _rows(state["k"], state["table"], n, count).transpose(2, 3))
    live = torch.arange(count, device="cuda") < (lens - n)[:, None]
    y = y.masked_fill(~live[:, None, None], -math.inf)
    p, total, top = _softmax(torch.cat((x, y), -1))
    x, y = p[..., :state["longest_shared"]], p[..., state["longest_shared"]:]
    stacked = x.new_zeros(groups, most, kvh, group, x.shape[-1])
    stacked[mine, place] = x
    o = torch.matmul(stacked.transpose(1, 2).flatten(2, 3), _rows(state["v"], table, zero, state["longest_shared"]))
    o = o.view(groups, kvh, most, group, DIM).transpose(1, 2)[mine, place]
    o = o + torch.matmul(y, _rows(state["v"], state["table"], n, count))
    return _finish(state, o, total, top)


# -------------------------------------------------------------------- the work --
def work(case):
    kvh, heads, seqs = case["kv_heads"], case["kv_heads"] * case["group"], case["seqs"]
    lens = _lens(case)
    if case["kind"] == "append":
        n = sum(_new(case))
        wide = 4 if case["input"] == "f32" else 2
        return {"bytes": n * (heads + 2 * kvh) * DIM * (wide + 2), "flops": 3.0 * n * (heads + kvh) * case["rotated"]}
    ends = seqs * heads * (ROW + DIM * (4 if case["out"] == "f32" else 2) + 4)
    if case["kind"] == "shared":
        shares = [m if n >= m else 0 for n, m in zip(lens, _per_seq(case))]
        cuts = _groups(case)
        once = sum(max(shares[a:b]) for a, b in zip(cuts, cuts[1:]))
        rows = once + sum(n - m for n, m in zip(lens, shares))
        return {"bytes": rows * kvh * 2 * ROW + ends, "flops": 4.0 * DIM * heads * sum(lens)}
    rows = sum(lens) - (sum(_first(case)) if case["first"] else 0)
    if case["prior"]:
        ends += seqs * heads * (4 * DIM + 4)
    return {"bytes": rows * kvh * 2 * ROW + ends, "flops": 4.0 * DIM * heads * rows}


# --------------------------------------------------- the definitions, in 64 bits --
def exact(case, seed):
    state = prepare(case, seed)
    page = case["page"]
    if case["kind"] == "append":
        half = case["rotated"] // 2
        unit = lambda pos: torch.polar(torch.ones(len(pos), half, dtype=torch.float64, device="cuda"),  # noqa: E731
                                       pos.double()[:, None] * state["freq"].double()[None])[:, None]
        pairs = torch.arange(2 * half, device="cuda").view(half, 2) if state["adjacent"] else torch.arange(2 * half, device="cuda").view(2, half).T

        def turned(x, pos):
            x = x.double().clone()
            z = torch.complex(x[..., pairs[:, 0]], x[..., pairs[:, 1]]) * unit(pos)
            x[..., pairs[:, 0]], x[..., pairs[:, 1]] = z.real, z.imag
            return x

        k, v, at, qs = state["k"].double(), state["v"].double(), 0, []
        for s, (n, m) in enumerate(zip(_lens(case), _new(case))):
            pos = torch.arange(n - m, n, device="cuda")
            pages = state["table"][s].long()[torch.div(pos, page, rounding_mode="floor")]
            k[pages, :, pos.remainder(page)] = turned(state["k_new"][at:at + m], pos)
            v[pages, :, pos.remainder(page)] = state["v_new"][at:at + m].double()
            qs.append(turned(state["q_new"][at:at + m], pos))
            at += m
        return torch.cat(qs), k, v
    heads, group = state["q"].shape[1], case["group"]
    firsts = _first(case) if case.get("first") else [0] * case["seqs"]
    outs, lses = [], []
    for s, n in enumerate(_lens(case)):
        q = state["q"][s].double()
        parts = []  # per stretch of rows: log of the sum of exp(score), mean value, per head
        for a in range(firsts[s], n, 16384):
            b = min(n, a + 16384)
            pages = state["table"][s, a // page:(b + page - 1) // page].long()
            cut = slice(a % page, a % page + b - a)
            kk = state["k"][pages].double().transpose(0, 1).reshape(case["kv_heads"], -1, DIM)[:, cut]
            vv = state["v"][pages].double().transpose(0, 1).reshape(case["kv_heads"], -1, DIM)[:, cut]
            kk, vv = kk.repeat_interleave(group, 0), vv.repeat_interleave(group, 0)
            score = (kk @ q[:, :, None])[..., 0] * DIM ** -0.5
            parts.append((torch.logsumexp(score, 1), (torch.softmax(score, 1)[:, None] @ vv)[:, 0]))
        if case.get("prior"):
            parts.append((state["prior"][1][s].double(), state["prior"][0][s].double()))
        if not parts:
            parts.append((torch.full((heads,), -math.inf, dtype=torch.float64, device="cuda"),
                          torch.zeros(heads, DIM, dtype=torch.float64, device="cuda")))
        logs, means = torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])
        lse = torch.logsumexp(logs, 0)
        share = torch.exp(logs - lse.clamp(min=-1e300))
        outs.append((share[:, :, None] * means).sum(0))
        lses.append(lse)
    return torch.stack(outs), torch.stack(lses)
