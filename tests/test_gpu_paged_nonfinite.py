"""Attention over a paged cache where scores, priors or values are not finite: a head whose softmax has no value is NaN, in
its output and in its lse, and never taken for a head without rows; all other heads are as without it."""
import numpy as np
import pytest
import torch

import paged as P
from test_gpu_paged import Buffers, freqs_of, only_dim_7, paged, q_dev, queries, shared_decode, shared_pool, wide_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dp():
    import paper_2602_05191_amd as dp
    return dp


NAN, INF, NINF, ONE, MINUS_ONE = P.NAN, 0x7F80, 0xFF80, 0x3F80, 0xBF80

# form of the call: lengths, layout, host bound of the lengths, shared rows of one group of all sequences
FORMS = {
    "whole": ([300, 37, 0, 1], "head", None, 0),          # a workgroup per segment
    "split": ([5000, 700, 0, 1], "head", None, 0),        # pieces of segments, merged
    "together": ([700, 333, 0, 1], "token", 0, 0),        # four KV heads per workgroup
    "shared": ([300, 237, 0, 201], "head", None, 200),    # the shared rows once
    "apart": ([300, 237, 0, 201], "head", None, -200),    # every sequence for itself
}


def make(dp, form, group=4, page=16, seed=60):
    lens, layout, bound, shared = FORMS[form]
    n_kv = 4 if form == "together" else 2
    if shared:
        pool = shared_pool([0, len(lens)], [abs(shared)], [max(0, n - abs(shared)) for n in lens], n_kv, page, seed=seed, idle={2})
    else:
        pool = P.Pool(lens, n_kv, page, seed=seed)
    if bound is not None:
        bound, width = wide_bound(len(lens), n_kv, page)
        pool.table = np.pad(pool.table, ((0, 0), (0, max(0, width - pool.table.shape[1]))), constant_values=-1)
    q = queries(pool.rng, len(lens), n_kv * group)

    def run(q, dtype=torch.float32, **kw):
        if shared:
            return shared_decode(dp, pool, q, [0, len(lens)], [abs(shared)], once=shared > 0, dtype=dtype, max_len=bound, **kw)
        return paged(dp, pool, q, layout, dtype, max_len=bound, **kw)

    return pool, q, run


def rows_of(pool, s, r, kv):
    return pool.table[s, r // pool.page], kv, r % pool.page


def holders(pool, s, r):
    """The sequences that attend row r of sequence s (on a page that they share, or alone)."""
    return [t for t in range(len(pool.lens)) if pool.lens[t] > r and pool.table[t, r // pool.page] == pool.table[s, r // pool.page]]


def check_heads(got, ref, bad, dtype):
    """The heads of bad are NaN, output and lse; the others are the reference's."""
    out, lse = got
    b = torch.from_numpy(bad).cuda()
    assert torch.isnan(out[b]).all() and torch.isnan(lse[b]).all()
    P.check((out[~b], lse[~b]), (ref[0][~bad], ref[1][~bad]), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("group", [4, 20])
@pytest.mark.parametrize("form", list(FORMS))
def test_a_nan_query_or_key(dp, form, group, dtype):
    """Query heads that hold NaN, or infinities of both signs (products of random signs: a score of NaN or +inf among 300
    rows or more); a key row that holds NaN."""
    pool, q, run = make(dp, form, group)
    ref = P.decode(pool, q)
    odd = q.copy()
    odd[0, 1, 3], odd[1, group, 100], odd[3, 2, 0] = NAN, NAN, NAN
    odd[0, group - 1, [4, 5]] = INF, NINF
    bad = np.zeros(q.shape[:2], dtype=bool)
    bad[0, 1] = bad[1, group] = bad[3, 2] = bad[0, group - 1] = True
    odd[2, :, 9] = NAN    # a sequence without rows: nothing is attended, whatever its queries hold
    check_heads(run(odd, dtype), ref, bad, dtype)
    for s, r, kv in ((0, 0, 0), (0, 299, 1), (1, 30, 1)):
        at = rows_of(pool, s, r, kv)
        keep = pool.k[at].copy()
        pool.k[at][7] = NAN
        bad = np.zeros(q.shape[:2], dtype=bool)
        for t in holders(pool, s, r):
            bad[t, kv * group:(kv + 1) * group] = True
        check_heads(run(q, dtype), ref, bad, dtype)
        pool.k[at] = keep


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", list(FORMS))
def test_an_infinite_key(dp, form, dtype):
    """A key of +inf in one dimension: heads that are positive there score +inf (inf - inf: NaN), heads that are negative
    there score -inf, which is a row without weight."""
    pool, q, run = make(dp, form)
    q[:, 0::2, 7], q[:, 1::2, 7] = ONE, MINUS_ONE
    for s, r in ((0, 0), (0, 150), (1, 36), (0, 299)):
        at = rows_of(pool, s, r, 1)
        keep = pool.k[at].copy()
        pool.k[at][7] = INF
        bad = np.zeros(q.shape[:2], dtype=bool)
        for t in holders(pool, s, r):
            bad[t, 4:8:2] = True
        check_heads(run(q, dtype), P.decode(pool, q), bad, dtype)
        pool.k[at] = keep


@pytest.mark.parametrize("form", ["whole", "split", "together"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_prior_that_is_not_finite(dp, form, dtype):
    """prior_lse of NaN or +inf, beside rows and without any; a prior of finite weight beside rows that score NaN."""
    pool, q, run = make(dp, form)
    n, heads = q.shape[:2]
    prior = [pool.rng.standard_normal((n, heads, 128)).astype(np.float32), pool.rng.uniform(-5, 9, (n, heads)).astype(np.float32)]
    ref = P.decode(pool, q, prior=prior)
    bad = np.zeros((n, heads), dtype=bool)
    for s, h, x in ((0, 0, np.nan), (0, 5, np.inf), (1, 7, np.nan), (2, 1, np.nan), (2, 6, np.inf), (3, 3, np.inf)):
        prior[1][s, h], bad[s, h] = x, True
    check_heads(run(q, dtype, prior=prior), ref, bad, dtype)
    prior[1][bad] = 3.0
    ref = P.decode(pool, q, prior=prior)
    bad[:], bad[0, 2] = False, True
    q[0, 2, 50] = NAN
    check_heads(run(q, dtype, prior=prior), ref, bad, dtype)


def test_a_nan_key_is_appended_and_attended(dp):
    """What a model leaves that has lost its numbers stays to be seen: a NaN in a new key reaches the pages, rotated with
    its partner, and every head that attends the token."""
    pool = P.Pool([40, 3], 2, 16, seed=61, spare=1)
    pool.lens = pool.lens + 1
    c = pool.device(8)
    k, v = (torch.from_numpy(pool.rng.standard_normal((2, 2, 128))).to(torch.bfloat16).cuda() for _ in range(2))
    k[0, 1, 12] = float("nan")
    dp.dp_append_kv(c, k, v, torch.tensor(freqs_of(128), device="cuda"))
    q = queries(pool.rng, 2, 8)
    b = Buffers(2, 8, dp.dp_paged_workspace_bytes(c))
    dp.dp_paged_decode(c, q_dev(q), b.out.t, b.lse.t, b.ws.t)
    out, lse = b.done()
    bad = torch.zeros(2, 8, dtype=torch.bool, device="cuda")
    bad[0, 4:] = True
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.isfinite(out[~bad]).all() and torch.isfinite(lse[~bad]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lead", [60.0, 99.0, 100.0, 110.0, 118.0, 125.0, 125.5])
@pytest.mark.parametrize("form", list(FORMS))
def test_an_infinite_value_of_little_weight(dp, form, lead, dtype):
    """One row leads all others by 60 to 125.5 in base 2 (a weight that is a power of two leaves nothing of itself for a second
    piece); an infinite value in front of it, next to it and far behind it stays in its dimension: +inf there, in all heads
    that attend the row, nothing elsewhere."""
    pool, q, run = make(dp, form)
    leader, scale = int(pool.lens[0]) // 2, float(np.float32(np.log(2)))   # (times log2 e: 1 in fp32)
    only_dim_7(pool, q, lambda i: np.where(i == leader, lead, 0.0))
    ref = P.decode(pool, q, scale=scale)
    for r in (0, leader + 1, int(pool.lens[0]) - 1):
        at = rows_of(pool, 0, r, 1)
        keep = pool.v[at].copy()
        pool.v[at][5] = INF
        out, lse = run(q, dtype, sm_scale=scale)
        for t in holders(pool, 0, r):
            assert torch.isposinf(out[t, 4:8, 5]).all()
            out[t, 4:8, 5] = torch.from_numpy(ref[0][t, 4:8, 5]).to(out)
        P.check((out, lse), ref, dtype)
        pool.v[at] = keep


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", list(FORMS))
def test_large_values_without_weight(dp, form, dtype):
    """Rows that score -inf hold the largest numbers there are: no trace of them."""
    pool, q, run = make(dp, form)
    q[..., 7] = ONE
    for r in (0, 33, 150, 299):
        at = rows_of(pool, 0, r, 1)
        pool.k[at][7], pool.v[at] = NINF, 0x7F7F
    P.check(run(q, dtype), P.decode(pool, q), dtype)
