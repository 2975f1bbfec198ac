"""Shared helpers of the tests of the paged cache: a pool with rubbish wherever nothing is stored, and the operators from
their formulas in 64 bits (numpy).  (Not a test module.)"""
from __future__ import annotations

import numpy as np
import torch

DIM = 128
NAN = 0x7FC1       # bf16 bits: what the places of a pool that hold nothing are filled with
BF16_HALF = 2.0 ** -8   # a rounding to bf16 is off by at most this, relative to the value


def bits(x: torch.Tensor) -> np.ndarray:
    return x.contiguous().cpu().view(torch.int16).numpy().view(np.uint16)


def wide(x) -> np.ndarray:
    """bf16 bits (or a tensor) as float64."""
    if isinstance(x, torch.Tensor):
        return x.detach().cpu().double().numpy()
    return (np.asarray(x, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bf16_bits(x: np.ndarray) -> np.ndarray:
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


class Pool:
    """A paged cache on the host: lens[s] tokens per sequence in pages handed out in no order, bf16 bits; every other
    place of the pool, the rest of a sequence's last page included, is NaN.  k, v: [n_pages, n_kv, page, 128]."""

    def __init__(self, lens, n_kv=1, page=16, seed=0, extra=3, width=None, spare=0, k_scale=1.0):
        self.rng = np.random.default_rng(seed)
        self.lens, self.n_kv, self.page = np.asarray(lens, dtype=np.int32), n_kv, page
        need = [-(-(int(n) + spare) // page) for n in lens]
        self.n_pages = sum(need) + extra
        order = self.rng.permutation(self.n_pages)
        self.table = np.full((len(lens), max(max(need + [0]), 1) if width is None else width), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, n_kv, page, DIM)
        self.k, self.v = np.full(shape, NAN, dtype=np.uint16), np.full(shape, NAN, dtype=np.uint16)
        for s, n in enumerate(lens):
            self.put(s, 0, k_scale * self.rng.standard_normal((int(n), n_kv, DIM)), self.rng.standard_normal((int(n), n_kv, DIM)))

    def put(self, s, first, k, v):
        i = np.arange(first, first + len(k))
        p, slot = self.table[s, i // self.page], i % self.page
        self.k[p, :, slot], self.v[p, :, slot] = to_bf16_bits(k), to_bf16_bits(v)

    def rows(self, s, first, last):
        """float64 [n_kv, rows, 128] of the rows on pages that are there."""
        i = np.arange(first, max(first, last))
        p = self.table[s, i // self.page]
        i, p = i[(p >= 0) & (p < self.n_pages)], p[(p >= 0) & (p < self.n_pages)]
        return (wide(self.k[p, :, i % self.page]).transpose(1, 0, 2), wide(self.v[p, :, i % self.page]).transpose(1, 0, 2))

    def device(self, n_q, layout="head", max_len=None, sm_scale=0.0):
        """dp.PagedCache with the pool uploaded in the given layout (head: heads outermost in a page; token: tokens
        outermost; side: K and V of a page side by side, rows padded)."""
        import paper_2602_05191_amd as dp
        up = lambda a: torch.from_numpy(a.view(np.int16)).cuda()  # noqa: E731
        if layout == "token":
            k, v = (up(a.transpose(0, 2, 1, 3).copy()).transpose(1, 2) for a in (self.k, self.v))
        elif layout == "side":
            both = torch.full((self.n_pages, 2, self.n_kv, self.page, DIM + 8), NAN, dtype=torch.int16, device="cuda")
            both[:, 0, ..., :DIM], both[:, 1, ..., :DIM] = up(self.k), up(self.v)
            k, v = both[:, 0, ..., :DIM], both[:, 1, ..., :DIM]
        else:
            k, v = up(self.k), up(self.v)
        longest = int(max(self.lens.max(), 0)) if max_len is None else max_len
        return dp.PagedCache(k, v, torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lens).cuda(), longest, n_q,
                             sm_scale)


def attention(q, k, v, scale, prior=None):
    """One KV head: q [G, 128], k, v [rows, 128] in float64 -> (out [G, 128], lse [G]); prior = (out, lse) is joined."""
    with np.errstate(all="ignore"):
        x = scale * (q @ k.T)
        top = x.max(axis=1, initial=-np.inf) if prior is None else np.maximum(x.max(axis=1, initial=-np.inf), prior[1])
        sub = np.where(np.isfinite(top), top, 0.0)[:, None]
        w = np.exp(x - sub)
        o = np.zeros((len(q), DIM))
        for g in range(len(q)):   # (a row without weight takes no part, whatever it holds)
            o[g] = (w[g, w[g] > 0, None] * v[w[g] > 0]).sum(0)
        z = w.sum(1)
        if prior is not None:
            p = np.exp(prior[1] - sub[:, 0])
            o, z = o + np.where(p > 0, p, 0.0)[:, None] * np.where(p[:, None] > 0, prior[0], 0.0), z + p
        return np.where(z[:, None] > 0, o / np.where(z > 0, z, 1)[:, None], 0.0), np.where(z > 0, np.log(z) + sub[:, 0], -np.inf)


def decode(pool, q, first=None, prior=None, scale=DIM ** -0.5):
    """q bf16 bits [n_seqs, n_q, 128] -> (out, lse) float64."""
    n, heads = q.shape[:2]
    group = heads // pool.n_kv
    out, lse = np.zeros((n, heads, DIM)), np.zeros((n, heads))
    for s in range(n):
        k, v = pool.rows(s, 0 if first is None else max(0, int(first[s])), max(0, int(pool.lens[s])))
        for h in range(pool.n_kv):
            cut = slice(h * group, (h + 1) * group)
            out[s, cut], lse[s, cut] = attention(wide(q[s, cut]), k[h], v[h], scale,
                                                 None if prior is None else (prior[0][s, cut], prior[1][s, cut]))
    return out, lse


def rotate(x, pos, freqs, adjacent):
    """x float64 [n, heads, 128] turned to positions pos [n] by pairs."""
    x, half = np.array(x, dtype=np.float64), len(freqs)
    t = (np.asarray(pos, dtype=np.float64)[:, None] * np.asarray(freqs, dtype=np.float64))[:, None]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if adjacent else (slice(0, half), slice(half, 2 * half))
    xa, xb = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = xa * np.cos(t) - xb * np.sin(t), xa * np.sin(t) + xb * np.cos(t)
    return x


def turned_close(got_bits, x, pos, freqs, adjacent):
    """Whether rotated rows are the exact ones up to one rounding to bf16 and fp32 arithmetic on a pair: two products and
    a sum (2^-24 each), sine and cosine to 2 units (2^-22 together), of a pair's length."""
    want = rotate(x, pos, freqs, adjacent)
    length = np.abs(x).max(axis=-1, keepdims=True) * 2 ** 0.5
    return (np.abs(wide(got_bits) - want) <= BF16_HALF * np.abs(want) + 8 * 2.0 ** -23 * length).all()


def check(got, want, dtype=torch.float32, tol=2e-5):
    """(out, lse) of a call against float64.  tol: fp32 sums of weighted values of size ~1 whose weights sum to 1 (a few
    2^-24 times the square root of the rows), above it the scores' own rounding, 2^-23 of their size (up to ~40)."""
    out, lse = (x.detach().float().cpu().numpy().astype(np.float64).reshape(w.shape) for x, w in zip(got, want))
    ref, ref_lse = want
    rounding = BF16_HALF if dtype == torch.bfloat16 else 0.0
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref_lse))
    assert (np.abs(out - ref) <= tol * np.maximum(1.0, np.abs(ref)) + rounding * np.abs(ref)).all(), np.abs(out - ref).max()
    fin = np.isfinite(ref_lse)
    assert (np.abs(lse[fin] - ref_lse[fin]) <= tol * np.maximum(1.0, np.abs(ref_lse[fin]))).all()
    assert (out[~fin] == 0).all()
