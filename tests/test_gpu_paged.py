"""GPU parity of the operators over a paged cache against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

import harness as H
import paged as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dp():
    import paper_2602_05191_amd as dp
    return dp


def up(a, dt=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).cuda()


def queries(rng, *shape, scale=1.0):
    return P.to_bf16_bits(scale * rng.standard_normal((*shape, 128)))


def q_dev(q):
    return torch.from_numpy(q.view(np.int16)).cuda().view(torch.bfloat16)


class Buffers:
    """Output and workspace between canaries; the workspace starts as NaN."""

    def __init__(self, n_seqs, n_q, ws_bytes, dtype=torch.float32):
        self.out = H.Guarded((n_seqs, n_q, 128), dtype, float("nan"))
        self.lse = H.Guarded((n_seqs, n_q), torch.float32, float("nan"))
        self.ws = H.Guarded((max(ws_bytes, 256),), torch.uint8, 0xFF)

    def done(self):
        torch.cuda.synchronize()
        for g, what in ((self.out, "out"), (self.lse, "lse"), (self.ws, "workspace")):
            g.check(what)
        return self.out.t, self.lse.t


def paged(dp, pool, q, layout="head", dtype=torch.float32, first=None, prior=None, max_len=None, sm_scale=0.0):
    c = pool.device(q.shape[1], layout, max_len, sm_scale)
    b = Buffers(*q.shape[:2], dp.dp_paged_workspace_bytes(c), dtype)
    kw = {} if prior is None else dict(prior_out=up(prior[0], np.float32), prior_lse=up(prior[1], np.float32))
    dp.dp_paged_decode(c, q_dev(q), b.out.t, b.lse.t, b.ws.t, first_rows=None if first is None else up(first), **kw)
    return b.done()


# ------------------------------------------------------------------ append --
def run_append(dp, pool, k, v, freqs, layout="head", q=None, ptr=None, positions=None, adjacent=False, dtype=torch.bfloat16,
               max_len=None, n_q=4):
    """Appends k, v (float64 [n, heads, 128]) as slices of one projection; -> (pool before, pool after) as bits, q_out bits
    and the values that the kernel was given, widened."""
    n, n_kv = k.shape[:2]
    heads = 0 if q is None else q.shape[1]
    x = torch.from_numpy(np.concatenate([k, v] + ([] if q is None else [q]), axis=1)).to(dtype).cuda()
    c = pool.device(n_q if q is None else heads, layout, max_len)
    before = P.bits(c.k_pages), P.bits(c.v_pages)
    out = H.Guarded((n, max(heads, 1), 128), torch.bfloat16, -3.0)
    f = None if freqs is None else torch.tensor(freqs, dtype=torch.float32, device="cuda")
    dp.dp_append_kv(c, x[:, :n_kv], x[:, n_kv:2 * n_kv], f, q=None if q is None else x[:, 2 * n_kv:],
                    q_out=None if q is None else out.t, tok_ptr=None if ptr is None else up(ptr),
                    positions=None if positions is None else up(positions), adjacent_pairs=adjacent)
    torch.cuda.synchronize()
    out.check("q_out")
    given = P.wide(x)
    return before, (P.bits(c.k_pages), P.bits(c.v_pages)), P.bits(out.t), (given[:, :n_kv], given[:, n_kv:2 * n_kv], given[:, 2 * n_kv:])


def freqs_of(rot):
    return (10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)


def check_append(before, after, q_out, given, pool, lens, ptr, freqs, adjacent, positions=None, max_len=None):
    k, v, q = given
    want_k, want_v = before[0].copy(), before[1].copy()
    touched = np.zeros(want_k.shape[:3], dtype=bool)
    exact = P.to_bf16_bits(v)
    for s in range(len(lens)):
        for t in range(ptr[s], ptr[s + 1]):
            at = int(lens[s]) - (ptr[s + 1] - t)
            pos = at if positions is None else positions[t]
            if q.shape[1]:
                assert P.turned_close(q_out[t:t + 1], q[t:t + 1], [pos], freqs, adjacent)
            page = pool.table[s, at // pool.page] if 0 <= at < (pool.table.shape[1] * pool.page if max_len is None else max_len) else -1
            if not 0 <= page < pool.n_pages:
                continue
            slot = at % pool.page
            assert P.turned_close(after[0][page, :, slot][None], k[t:t + 1], [pos], freqs, adjacent)
            want_k[page, :, slot], want_v[page, :, slot] = after[0][page, :, slot], exact[t]
    assert np.array_equal(after[0], want_k) and np.array_equal(after[1], want_v)   # (nothing else of the pool is written)


@pytest.mark.parametrize("layout", ["head", "token", "side"])
@pytest.mark.parametrize("page, n_kv, n_q", [(1, 1, 1), (16, 2, 10), (64, 8, 32)])
@pytest.mark.parametrize("dtype, rot, adjacent", [(torch.bfloat16, 128, False), (torch.bfloat16, 48, True),
                                                  (torch.float32, 64, False), (torch.float32, 128, True),
                                                  (torch.bfloat16, 0, False)])
def test_append(dp, layout, page, n_kv, n_q, dtype, rot, adjacent):
    """Several sequences, some without new tokens, new tokens over page borders and at the very beginning."""
    lens, new = [5, 1, 130, 0, 64, 17], [5, 1, 90, 0, 1, 0]
    ptr = np.concatenate([[0], np.cumsum(new)])
    pool = P.Pool(lens, n_kv, page, seed=rot + page)
    rng = pool.rng
    k, v, q = (rng.standard_normal((int(ptr[-1]), h, 128)) for h in (n_kv, n_kv, n_q))
    f = freqs_of(rot)
    r = run_append(dp, pool, k, v, f if rot else None, layout, q, ptr, None, adjacent, dtype)
    check_append(*r, pool, lens, ptr, f, adjacent)


@pytest.mark.parametrize("n_seqs", [1, 2, 64, 65, 300])
def test_append_of_one_token_each(dp, n_seqs):
    """Without a list of tokens, and the same with one: a search over more sequences than a wave has lanes."""
    rng = np.random.default_rng(n_seqs)
    lens = rng.integers(1, 40, n_seqs)
    ptr = np.arange(n_seqs + 1)
    f = freqs_of(128)
    k, v, q = (rng.standard_normal((n_seqs, h, 128)) for h in (2, 2, 6))
    results = []
    for p in (None, ptr):
        pool = P.Pool(lens, 2, 8, seed=3)
        r = run_append(dp, pool, k, v, f, q=q, ptr=p)
        check_append(*r, pool, lens, ptr, f, False)
        results.append(r)
    for a, b in zip(results[0][1] + (results[0][2],), results[1][1] + (results[1][2],)):
        assert np.array_equal(a, b)


def test_append_finds_the_sequence_of_every_token(dp):
    """5000 sequences with 0 to 3 new tokens, runs of sequences without any, tokens in front of the first and behind the last."""
    rng = np.random.default_rng(9)
    new = rng.integers(0, 4, 5000)
    new[100:900] = 0
    new[-70:] = 0
    lens = new + rng.integers(0, 5, 5000)
    ptr = 3 + np.concatenate([[0], np.cumsum(new)])
    n = int(ptr[-1]) + 5
    pool = P.Pool(lens, 1, 4, seed=9)
    k, v, q = (rng.standard_normal((n, 1, 128)) for _ in range(3))
    f = freqs_of(32)
    r = run_append(dp, pool, k, v, f, q=q, ptr=ptr)
    check_append(*r, pool, lens, ptr, f, False)
    outside = np.concatenate([r[2][:3], r[2][-5:]])
    assert (outside == P.to_bf16_bits(np.array([-3.0]))[0]).all()   # tokens that no sequence holds: q_out as it was


@pytest.mark.parametrize("position", [0, 131071, 2 ** 24 + 1, 2 ** 31 - 1, -7])
@pytest.mark.parametrize("adjacent", [False, True])
def test_append_far_positions(dp, position, adjacent):
    lens, ptr = [9, 3], [0, 1, 2]
    pool = P.Pool(lens, 2, 16, seed=4)
    rng = pool.rng
    k, v, q = (rng.standard_normal((2, h, 128)) for h in (2, 2, 4))
    f = np.concatenate([[1.0, 3.7], freqs_of(128)[2:]]).astype(np.float32)
    pos = np.array([position, max(position - 1, -8)])
    r = run_append(dp, pool, k, v, f, q=q, ptr=ptr, positions=pos, adjacent=adjacent, dtype=torch.float32)
    check_append(*r, pool, lens, ptr, f, adjacent, positions=pos)


def test_append_leaves_out_what_has_no_place(dp):
    """Pages that are not there, places in front of the first row and behind max_seq_len: q_out is written, the pool is not."""
    lens, new = [20, 3, 40, 50], [4, 5, 12, 20]
    pool = P.Pool(lens, 2, 8, seed=6)
    pool.table[0, 2], pool.table[2, 4] = -1, pool.n_pages
    pool.table[3, 5] = 2 ** 31 - 1
    ptr = np.concatenate([[0], np.cumsum(new)])
    k, v, q = (pool.rng.standard_normal((int(ptr[-1]), h, 128)) for h in (2, 2, 4))
    f = freqs_of(128)
    r = run_append(dp, pool, k, v, f, q=q, ptr=ptr, max_len=45)
    check_append(*r, pool, lens, ptr, f, False, max_len=45)
    assert (r[2] != P.to_bf16_bits(np.array([-3.0]))[0]).any(axis=(1, 2)).all()
    # a pool without a page, a cache without a row
    none = P.Pool([0, 0], 2, 8, seed=6, extra=0)
    c = none.device(4, max_len=0)
    x = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    dp.dp_append_kv(c, x, x)
    torch.cuda.synchronize()


def test_append_keys_and_values_only_and_queries_in_place(dp):
    lens = [33, 2, 7]
    f = freqs_of(128)
    pool = P.Pool(lens, 2, 16, seed=7)
    k, v, q = (pool.rng.standard_normal((3, h, 128)) for h in (2, 2, 6))
    r = run_append(dp, pool, k, v, f)
    check_append(*r, pool, lens, [0, 1, 2, 3], f, False)
    c = pool.device(6)
    kd, vd, qd = (torch.from_numpy(a).to(torch.bfloat16).cuda() for a in (k, v, q))
    other, given = torch.empty_like(qd), P.wide(qd)
    fd = torch.tensor(f, device="cuda")
    dp.dp_append_kv(c, kd, vd, fd, q=qd, q_out=other)
    dp.dp_append_kv(c, kd, vd, fd, q=qd, q_out=qd)
    torch.cuda.synchronize()
    assert np.array_equal(P.bits(other), P.bits(qd)) and P.turned_close(P.bits(qd), given, [32, 1, 6], f, False)


def test_append_writes_queries_between_what_it_reads(dp):
    """q_out in the gap between two tokens' rows of q, k and v; one strided token in place; neither touches a row that is read."""
    pool = P.Pool([9, 5], 2, 16, seed=46)
    c, f = pool.device(6), torch.tensor(freqs_of(128), device="cuda")
    x = torch.from_numpy(pool.rng.standard_normal((2, 40, 128))).to(torch.bfloat16).cuda()
    q, k, v, gap = x[:, :6], x[:, 6:8], x[:, 8:10], x[0, 20:32].view(2, 6, 128)
    want, given = torch.empty(2, 6, 128, dtype=torch.bfloat16, device="cuda"), x.clone()
    dp.dp_append_kv(c, k, v, f, q=q, q_out=want)
    stored = c.k_pages.clone(), c.v_pages.clone()
    dp.dp_append_kv(c, k, v, f, q=q, q_out=gap)
    torch.cuda.synchronize()
    assert torch.equal(gap, want) and torch.equal(c.k_pages, stored[0]) and torch.equal(c.v_pages, stored[1])
    given[0, 20:32] = want.view(12, 128)
    assert torch.equal(x, given)
    one = P.Pool([9], 2, 16, seed=47).device(6)
    dp.dp_append_kv(one, k[:1], v[:1], f, q=q[:1], q_out=q[:1])
    torch.cuda.synchronize()
    given[0, :6] = want[0]
    assert torch.equal(x, given)
    with pytest.raises(dp.DPError):
        dp.dp_append_kv(c, k, v, f, q=x[:, 28:34], q_out=gap)   # (the first token's heads of this q lie in the gap)


def test_append_of_many_tokens_is_the_append_of_its_parts(dp):
    """A prompt beyond 256 MiB of rows (written past the caches) and the same one in three parts (which are not): same bits."""
    n, n_kv, n_q, page = 120000, 2, 6, 64
    x = torch.randn(n, n_q + 2 * n_kv, 128, device="cuda", dtype=torch.bfloat16, generator=torch.Generator("cuda").manual_seed(1))
    q, k, v = x[:, :n_q], x[:, n_q:n_q + n_kv], x[:, n_q + n_kv:]
    f = torch.tensor(freqs_of(128), device="cuda")
    table = torch.randperm(n // page, generator=torch.Generator().manual_seed(2)).int().cuda()[None]
    results = []
    for cuts in ([0, n], [0, 50000, 50001, n]):
        pages = torch.zeros(2, n // page, n_kv, page, 128, device="cuda", dtype=torch.bfloat16)
        lens = torch.zeros(1, device="cuda", dtype=torch.int32)
        c = dp.PagedCache(pages[0], pages[1], table, lens, n, n_q)
        out = torch.empty(n, n_q, 128, device="cuda", dtype=torch.bfloat16)
        for a, b in zip(cuts, cuts[1:]):
            lens.fill_(b)
            dp.dp_append_kv(c, k[a:b], v[a:b], f, q=q[a:b], q_out=out[a:b], tok_ptr=up([0, b - a]))
        results.append((pages, out))
    torch.cuda.synchronize()
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    at = [0, 77777, n - 1]
    assert P.turned_close(P.bits(results[0][1][at]), P.wide(q[at]), at, freqs_of(128), False)


def test_append_of_many_fp32_tokens_is_the_append_of_its_parts(dp):
    """The same from fp32, pairs side by side, into pages with the tokens outermost, keys and values in strides of their own."""
    n, n_kv, n_q, page = 130000, 4, 4, 16
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(n, n_q + n_kv + 1, 128, device="cuda", generator=gen)
    v = torch.randn(n, n_kv, 128, device="cuda", generator=gen)
    q, k = x[:, :n_q], x[:, n_q:n_q + n_kv]
    f = torch.tensor(freqs_of(96), device="cuda")
    table = torch.randperm(n // page, generator=torch.Generator().manual_seed(4)).int().cuda()[None]
    results = []
    for cuts in ([0, n], [0, 60000, 60007, n]):
        pages = torch.zeros(2, n // page, page, n_kv, 128, device="cuda", dtype=torch.bfloat16)
        lens = torch.zeros(1, device="cuda", dtype=torch.int32)
        c = dp.PagedCache(pages[0].transpose(1, 2), pages[1].transpose(1, 2), table, lens, n, n_q)
        out = torch.empty(n, n_q, 128, device="cuda", dtype=torch.bfloat16)
        for a, b in zip(cuts, cuts[1:]):
            lens.fill_(b)
            dp.dp_append_kv(c, k[a:b], v[a:b], f, q=q[a:b], q_out=out[a:b], tok_ptr=up([0, b - a]), adjacent_pairs=True)
        results.append((pages, out))
    torch.cuda.synchronize()
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    at = [0, 88888, n - 1]
    assert P.turned_close(P.bits(results[0][1][at]), P.wide(q[at]), at, freqs_of(96), True)
    places = table[0, [i // page for i in at]].long().cpu().tolist()
    for i, p in zip(at, places):
        assert P.turned_close(P.bits(results[0][0][0, p, i % page][None]), P.wide(k[i:i + 1]), [i], freqs_of(96), True)
        assert torch.equal(results[0][0][1, p, i % page], v[i].to(torch.bfloat16))


def test_append_keeps_infinities_and_nan_in_their_pair(dp):
    lens, f = [5], freqs_of(64)
    for bad, dims in ((np.inf, (3, 35)), (np.nan, (3, 35)), (np.inf, (100,))):
        pool = P.Pool(lens, 1, 16, seed=8)
        k, v = pool.rng.standard_normal((1, 1, 128)), pool.rng.standard_normal((1, 1, 128))
        clean = run_append(dp, pool, k, v, f)
        k[0, 0, dims[0]], v[0, 0, 9] = bad, bad
        r = run_append(dp, pool, k, v, f)
        page, slot = pool.table[0, 0], 4
        got, was = P.wide(r[1][0][page, 0, slot]), P.wide(clean[1][0][page, 0, slot])
        odd = np.zeros(128, dtype=bool)
        odd[list(dims)] = True
        assert not np.isfinite(got[odd]).any() and np.array_equal(got[~odd], was[~odd])
        got = P.wide(r[1][1][page, 0, slot])
        assert np.array_equal(np.isnan(got), np.isnan(v[0, 0])) and not np.isfinite(got[9]) and np.isfinite(np.delete(got, 9)).all()


# ------------------------------------------------------------- paged decode --
EDGES = [0, 1, 15, 16, 17, 63, 64, 65, 129, 255, 320, 321, 700]


@pytest.mark.parametrize("n_kv, group", [(1, 1), (2, 4), (1, 5), (1, 16), (1, 20), (3, 7)])
@pytest.mark.parametrize("page, layout", [(1, "head"), (2, "token"), (8, "side"), (16, "head"), (64, "token"), (512, "side")])
def test_decode_at_edges(dp, n_kv, group, page, layout):
    pool = P.Pool(EDGES, n_kv, page, seed=page + group)
    q = queries(pool.rng, len(EDGES), n_kv * group)
    P.check(paged(dp, pool, q, layout), P.decode(pool, q))


@pytest.mark.parametrize("lens", [[3000, 1, 0, 777, 2049], [1500] * 40, [40000], [5, 9000, 0, 3], [2000] * 130, [64] * 600])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decode_splits(dp, lens, page, dtype):
    """Rows of a sequence over several workgroups, sequences of very different lengths, many sequences."""
    n_kv = 2 if sum(lens) < 50000 else 1
    pool = P.Pool(lens, n_kv, page, seed=len(lens), extra=0)
    q = queries(pool.rng, len(lens), 4 * n_kv, scale=1.5)
    P.check(paged(dp, pool, q, dtype=dtype), P.decode(pool, q), dtype)


@pytest.mark.parametrize("prior", [False, True])
@pytest.mark.parametrize("page", [4, 16, 64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decode_first_rows_and_prior(dp, prior, page, dtype):
    """First rows inside tiles and pages, behind the end, negative; a prior that weighs much, little or nothing."""
    lens = [700, 700, 64, 0, 90, 33, 2500, 1]
    first = [0, 333, 64, 5, 100, -3, 2477, 0]
    pool = P.Pool(lens, 2, page, seed=page)
    q = queries(pool.rng, len(lens), 8)
    p = None
    if prior:
        p = [pool.rng.standard_normal((len(lens), 8, 128)).astype(np.float32), pool.rng.uniform(-5, 15, (len(lens), 8)).astype(np.float32)]
        p[1][0, 0] = 300.0
        p[1][1, 3] = p[1][3, 2] = p[1][4, 7] = -np.inf
        p[0][1, 3] = p[0][3, 2] = np.nan    # (without weight: takes no part)
    P.check(paged(dp, pool, q, dtype=dtype, first=first, prior=p), P.decode(pool, q, first, p), dtype)


def test_decode_joins_in_place(dp):
    """prior_out = out and prior_lse = lse, in both forms (one workgroup per segment, split segments)."""
    for lens in ([100, 0, 7], [9000, 4000, 0]):
        pool = P.Pool(lens, 1, 16, seed=11)
        q = queries(pool.rng, 3, 4)
        prior = pool.rng.standard_normal((3, 4, 128)).astype(np.float32), pool.rng.uniform(2, 9, (3, 4)).astype(np.float32)
        c = pool.device(4)
        ws = torch.empty(dp.dp_paged_workspace_bytes(c), dtype=torch.uint8, device="cuda")
        out, lse = up(prior[0], np.float32), up(prior[1], np.float32)
        dp.dp_paged_decode(c, q_dev(q), out, lse, ws, prior_out=out, prior_lse=lse)
        torch.cuda.synchronize()
        P.check((out, lse), P.decode(pool, q, prior=prior))


def test_decode_leaves_out_pages_that_are_not_there(dp):
    for page in (4, 16, 64):
        pool = P.Pool([500, 130, 64, 3000], 1, page, seed=12)
        pool.table[0, [0, 3]] = -1, pool.n_pages
        pool.table[1, :] = -5
        pool.table[2, 0] = 2 ** 31 - 1
        pool.table[3, 5::7] = -2 ** 31
        q = queries(pool.rng, 4, 4)
        P.check(paged(dp, pool, q), P.decode(pool, q))


def test_decode_clamps_lengths(dp):
    pool = P.Pool([100, 40, 200], 1, 16, seed=13)
    q = queries(pool.rng, 3, 2)
    pool.lens = np.array([100, -4, 200], dtype=np.int32)
    got = paged(dp, pool, q, max_len=150)
    pool.lens = np.array([100, 0, 150], dtype=np.int32)
    P.check(got, P.decode(pool, q))
    none = P.Pool([0, 0], 2, 8, seed=6, extra=0)
    P.check(paged(dp, none, queries(none.rng, 2, 4), max_len=0), P.decode(none, queries(none.rng, 2, 4)))


@pytest.mark.parametrize("n", [1, 37, 64, 1000, 5000])
def test_decode_keeps_an_infinite_value_in_its_dimension(dp, n):
    pool = P.Pool([n], 1, 16, seed=14, k_scale=0.3)
    pool.v[pool.table[0, (n - 1) // 16], 0, (n - 1) % 16, 5] = H_INF
    q = queries(pool.rng, 1, 4)
    out, _ = paged(dp, pool, q)
    assert torch.isposinf(out[..., 5]).all() and torch.isfinite(out).sum() == out.numel() - 4


H_INF, H_NINF, H_ONE, H_LOWEST = 0x7F80, 0xFF80, 0x3F80, 0xFF7F


@pytest.mark.parametrize("low", [H_NINF, H_LOWEST])
@pytest.mark.parametrize("n, lo, hi", [(300, 64, 128), (300, 0, 16), (3000, 0, 2900), (37, 0, 37)])
def test_decode_rows_that_are_masked_by_their_score(dp, low, n, lo, hi):
    """Rows whose score is -inf, or the lowest number there is: no weight beside others; where all rows score -inf, none."""
    pool = P.Pool([n], 1, 16, seed=15, k_scale=0.3)
    q = queries(pool.rng, 1, 4)
    q[..., 7] = H_ONE
    for r in range(lo, hi):
        pool.k[pool.table[0, r // 16], 0, r % 16, 7] = low
    if low == H_LOWEST and lo == 0 and hi == n:
        # equal scores of -3.4e38 / 11.3 up to fp32 rounding of 3e37: any weights; only finite results are asked for
        out, lse = paged(dp, pool, q)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        return
    P.check(paged(dp, pool, q), P.decode(pool, q))


LOWEST = float(P.wide(np.array(H_LOWEST)))


def only_dim_7(pool, q, scores):
    """Keys and queries so that row i of every sequence scores exactly scores(i) at sm_scale = 1."""
    q[:], q[..., 7] = 0, H_ONE
    there = ~np.isnan(P.wide(pool.k))
    pool.k[there] = 0
    for s, n in enumerate(pool.lens):
        i = np.arange(n)
        pool.k[pool.table[s, i // pool.page], :, i % pool.page, 7] = P.to_bf16_bits(scores(i))[:, None]


@pytest.mark.parametrize("prior", [False, True])
@pytest.mark.parametrize("n", [37, 3000])
def test_decode_of_rows_that_score_the_lowest_numbers(dp, n, prior):
    """All rows at the lowest number there is: the mean; the lesser of two such scores has no weight (both forms)."""
    for scores in (lambda i: np.full(len(i), LOWEST), lambda i: np.where(i % 3 == 0, LOWEST, -2.0 ** 127)):
        pool = P.Pool([n, 11], 1, 16, seed=41)
        q = queries(pool.rng, 2, 4)
        only_dim_7(pool, q, scores)
        kw = {}
        if prior:
            kw["prior"] = pool.rng.standard_normal((2, 4, 128)).astype(np.float32), np.full((2, 4), LOWEST, np.float32)
        P.check(paged(dp, pool, q, sm_scale=1.0, **kw), P.decode(pool, q, scale=1.0, **kw))


def test_decode_sm_scale(dp):
    pool = P.Pool([333, 20], 1, 16, seed=16)
    q = queries(pool.rng, 2, 3)
    P.check(paged(dp, pool, q, sm_scale=0.03), P.decode(pool, q, scale=np.float64(np.float32(0.03))))


def test_places_beyond_32_bits(dp):
    """A pool of 4.5 GiB of keys (and of values): pages at its two ends, appended to and read."""
    n_pages, page, n_kv = 36 * 1024, 64, 8
    k = torch.empty(n_pages, n_kv, page, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    pool = P.Pool([150], n_kv, page, seed=17, extra=0)
    far = np.array([n_pages - 1, 0, n_pages - 2])
    for i, p in enumerate(far):
        k[p] = torch.from_numpy(pool.k[pool.table[0, i]].view(np.int16)).cuda().view(torch.bfloat16)
        v[p] = torch.from_numpy(pool.v[pool.table[0, i]].view(np.int16)).cuda().view(torch.bfloat16)
    c = dp.PagedCache(k, v, up(far[None]), up([151]), 160, 32)
    x, y = pool.rng.standard_normal((2, 1, n_kv, 128))
    dp.dp_append_kv(c, torch.from_numpy(x).to(torch.bfloat16).cuda(), torch.from_numpy(y).to(torch.bfloat16).cuda())
    pool.put(0, 150, x, y)
    pool.lens = np.array([151], dtype=np.int32)
    q = queries(pool.rng, 1, 32)
    b = Buffers(1, 32, dp.dp_paged_workspace_bytes(c))
    dp.dp_paged_decode(c, q_dev(q), b.out.t, b.lse.t, b.ws.t)
    P.check(b.done(), P.decode(pool, q))
    got = P.bits(k[n_pages - 2])
    assert np.array_equal(got[:, 150 - 128], pool.k[pool.table[0, 2]][:, 150 - 128])


@pytest.mark.parametrize("layout", ["head", "token"])
def test_decode_of_very_many_sequences(dp, layout):
    """More sequences than are dealt out (each is taken whole), some long, most short or empty."""
    rng = np.random.default_rng(18)
    lens = rng.integers(0, 24, 4200)
    lens[[0, 99, 4199]] = 900, 1, 1300
    pool = P.Pool(lens, 1, 16, seed=18)
    q = queries(pool.rng, len(lens), 2)
    P.check(paged(dp, pool, q, layout), P.decode(pool, q))


def wide_bound(n_seqs, n_kv, page):
    """max_len from which on four KV heads that lie side by side are read by one workgroup, and the table's width for it."""
    longest = -(-4096 // (n_seqs * n_kv)) * 64
    return longest, -(-longest // page)


@pytest.mark.parametrize("n_kv, group", [(4, 1), (8, 4), (4, 16), (4, 20), (12, 5)])
@pytest.mark.parametrize("page", [1, 8, 16, 64, 256])
def test_decode_of_heads_side_by_side(dp, n_kv, group, page):
    """Tokens outermost and a bound of many rows: four KV heads per workgroup.  First rows inside a tile, behind the end and
    negative, a prior for some heads, idle sequences, pages that are not there."""
    lens = [700, 17, 0, 1, 333, 64, 2049]
    first = [0, 16, 0, 0, 101, 64, -3]
    longest, width = wide_bound(len(lens), n_kv, page)
    longest = max(longest, 2049)
    pool = P.Pool(lens, n_kv, page, seed=51 + page, extra=0, width=max(width, -(-2049 // page)))
    pool.table[4, -(-150 // page)] = -7 if 150 + page < 333 else pool.table[4, -(-150 // page)]
    q = queries(pool.rng, len(lens), n_kv * group)
    prior = [pool.rng.standard_normal((len(lens), n_kv * group, 128)).astype(np.float32),
             pool.rng.uniform(-5, 9, (len(lens), n_kv * group)).astype(np.float32)]
    prior[1][1] = -np.inf
    P.check(paged(dp, pool, q, "token", first=first, prior=prior, max_len=longest), P.decode(pool, q, first, prior))
    got = paged(dp, pool, q, "token", max_len=longest)
    P.check(got, P.decode(pool, q))
    assert all(torch.equal(x, y) for x, y in zip(got, paged(dp, pool, q, "token", max_len=longest)))


@pytest.mark.parametrize("lens", [[40000], [9000, 3, 0, 20000], [1100] * 40])
def test_decode_of_heads_side_by_side_splits(dp, lens):
    """The same with rows enough for every workgroup; a bound beyond the lengths."""
    n_kv = 8 if len(lens) == 1 else 4
    pool = P.Pool(lens, n_kv, 16, seed=len(lens), extra=0, width=4096)
    q = queries(pool.rng, len(lens), 4 * n_kv, scale=1.5)
    P.check(paged(dp, pool, q, "token", torch.bfloat16, max_len=65536), P.decode(pool, q), torch.bfloat16)


@pytest.mark.parametrize("form", ["wide_table", "no_lse", "odd_out", "raw_bits"])
def test_forms_of_arguments(dp, form):
    """A table that is a slice of a wider one; no lse; an output at an odd element; queries and pages as raw bits."""
    pool = P.Pool([3000, 0, 70], 2, 16, seed=43)
    q = queries(pool.rng, 3, 8)
    c, Q = pool.device(8), q_dev(q)
    if form == "wide_table":
        wide = torch.full((3, c.page_table.shape[1] + 9), 1 << 30, dtype=torch.int32, device="cuda")
        table = wide[:, 4:4 + c.page_table.shape[1]]
        table.copy_(c.page_table)
        c = dp.PagedCache(c.k_pages, c.v_pages, table, c.seq_lens, 3000, 8)
    if form == "raw_bits":
        Q = Q.view(torch.int16)
    else:
        c = dp.PagedCache(c.k_pages.view(torch.bfloat16), c.v_pages.view(torch.bfloat16), c.page_table, c.seq_lens, 3000, 8)
    dtype = torch.bfloat16 if form == "odd_out" else torch.float32
    out = torch.full((3 * 8 * 128 + 1,), float("nan"), dtype=dtype, device="cuda")[1:].view(3, 8, 128)
    lse = None if form == "no_lse" else torch.empty(3, 8, device="cuda")
    ref = P.decode(pool, q)
    prefix = dp.SharedPrefix(up([0, 1]), up([100]), 1, 100, dp.DP_SHARED_PREFIX_ONCE)
    for call, n in ((dp.dp_paged_decode, dp.dp_paged_workspace_bytes(c)),
                    (dp.dp_shared_prefix_decode, dp.dp_shared_prefix_workspace_bytes(c, prefix))):
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        out.fill_(float("nan"))
        call(c, *([prefix] if call is dp.dp_shared_prefix_decode else []), Q, out, lse, ws)
        torch.cuda.synchronize()
        P.check((out, torch.from_numpy(ref[1]) if lse is None else lse), ref, dtype)


def test_a_pool_without_pages(dp):
    """Nothing is stored, nothing read; the prior passes through, queries are rotated."""
    pages = torch.empty(0, 2, 16, 128, dtype=torch.bfloat16, device="cuda")
    c = dp.PagedCache(pages, pages, torch.zeros(2, 4, dtype=torch.int32, device="cuda"), up([64, 3]), 64, 4)
    rng = np.random.default_rng(44)
    q = queries(rng, 2, 4)
    prior = torch.randn(2, 4, 128, device="cuda"), torch.randn(2, 4, device="cuda")
    b = Buffers(2, 4, dp.dp_paged_workspace_bytes(c))
    dp.dp_paged_decode(c, q_dev(q), b.out.t, b.lse.t, b.ws.t, prior_out=prior[0], prior_lse=prior[1])
    out, lse = b.done()
    # one weight, 2^(lse - lse): out = o / 1, lse = lse + ln 1
    assert torch.equal(out, prior[0]) and torch.equal(lse, prior[1])
    k, turned = q_dev(queries(rng, 2, 2)), torch.empty(2, 4, 128, dtype=torch.bfloat16, device="cuda")
    dp.dp_append_kv(c, k, k, q=q_dev(q), q_out=turned)
    torch.cuda.synchronize()
    assert np.array_equal(P.bits(turned), q)


def test_append_of_one_row_for_all(dp):
    """Keys and values with a stride of zero between tokens."""
    pool = P.Pool([0], 2, 16, seed=45, width=3, spare=40)
    k = torch.from_numpy(pool.rng.standard_normal((1, 2, 128))).float().cuda().expand(37, 2, 128)
    pool.lens[:] = 37
    c = pool.device(4)
    dp.dp_append_kv(c, k, k, tok_ptr=up([0, 37]))
    torch.cuda.synchronize()
    want = P.to_bf16_bits(k[0].cpu().numpy())
    for i in range(37):
        for pages in (c.k_pages, c.v_pages):
            assert np.array_equal(P.bits(pages[int(pool.table[0, i // 16]), :, i % 16]), want)


# ------------------------------------------------------------ shared prefix --
def shared_pool(ptr, shared, own_rows, n_kv, page, seed, idle=()):
    """Sequences of groups that begin alike: whole pages inside the shared rows are the same pages.  own_rows: rows of
    each sequence behind them; idle: sequences of no rows."""
    group = np.searchsorted(np.asarray(ptr), np.arange(len(own_rows)), side="right") - 1
    of = lambda s: int(shared[group[s]]) if 0 <= group[s] < len(shared) else 0  # noqa: E731
    lens = [0 if s in idle else of(s) + n for s, n in enumerate(own_rows)]
    pool = P.Pool(lens, n_kv, page, seed=seed)
    for g in range(len(shared)):
        users = [s for s in range(max(ptr[g], 0), min(ptr[g + 1], len(lens))) if lens[s]]
        whole = shared[g] // page
        for s in users[1:]:
            k, v = pool.rows(users[0], 0, shared[g])
            pool.put(s, 0, k.transpose(1, 0, 2), v.transpose(1, 0, 2))
            pool.table[s, :whole] = pool.table[users[0], :whole]
    return pool


def shared_decode(dp, pool, q, ptr, shared, most=None, longest=None, layout="head", dtype=torch.float32, max_len=None, once=True,
                  sm_scale=0.0):
    """once: the shared rows read once whatever the sizes (small calls attend every sequence for itself)."""
    c = pool.device(q.shape[1], layout, max_len, sm_scale)
    most = int(max(np.diff(ptr).max(), 1)) if most is None else most
    prefix = dp.SharedPrefix(up(ptr), up(shared), most, int(max(max(shared), 0)) if longest is None else longest,
                             dp.DP_SHARED_PREFIX_ONCE if once else 0)
    b = Buffers(*q.shape[:2], dp.dp_shared_prefix_workspace_bytes(c, prefix), dtype)
    dp.dp_shared_prefix_decode(c, prefix, q_dev(q), b.out.t, b.lse.t, b.ws.t)
    return b.done()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("page, layout", [(1, "head"), (8, "token"), (16, "side"), (64, "head"), (256, "token")])
@pytest.mark.parametrize("n_kv, group", [(1, 1), (2, 4), (1, 7), (1, 16), (1, 20)])
def test_shared_groups(dp, dtype, page, layout, n_kv, group):
    """Groups of 1, 2, 9 and 0 sequences, shared rows of 1 to 700, own rows from none on, idle slots (the first of a group
    among them)."""
    ptr, shared = [0, 1, 3, 12, 12], [33, 700, 129, 64]
    own = [5, 0, 70, 1, 9, 0, 33, 64, 65, 128, 2, 300]
    pool = shared_pool(ptr, shared, own, n_kv, page, seed=page + group, idle={3, 6})
    q = queries(pool.rng, len(own), n_kv * group, scale=1.5)
    ref = P.decode(pool, q)
    P.check(shared_decode(dp, pool, q, ptr, shared, layout=layout, dtype=dtype), ref, dtype)
    P.check(shared_decode(dp, pool, q, ptr, shared, layout=layout, dtype=dtype, once=False), ref, dtype)


def test_shared_rows_are_read_once_where_that_saves_much(dp):
    """9 sequences that share 20000 rows of 2 KV heads (164 MB of reads saved, 88 are asked for): told apart from the other
    form by a sequence whose own table lacks the shared pages."""
    pool = shared_pool([0, 9], [20000], [30] * 9, 2, 64, seed=20)
    q = queries(pool.rng, 9, 8)
    ref = P.decode(pool, q)
    pool.table[5, :20000 // 64] = -1
    P.check(shared_decode(dp, pool, q, [0, 9], [20000], once=False), ref)


@pytest.mark.parametrize("n_seqs", [2, 8, 16, 17, 33, 70, 150])
@pytest.mark.parametrize("shared", [1, 31, 32, 64, 65, 500, 6000])
def test_shared_columns_and_rows(dp, n_seqs, shared):
    """One group, whatever fills the columns of a tile and the rows of a block."""
    rng = np.random.default_rng(n_seqs)
    pool = shared_pool([0, n_seqs], [shared], list(rng.integers(0, 90, n_seqs)), 1, 16, seed=shared)
    q = queries(pool.rng, n_seqs, 4, scale=1.5)
    P.check(shared_decode(dp, pool, q, [0, n_seqs], [shared]), P.decode(pool, q))


def test_shared_prefix_is_the_paged_decode(dp):
    """Sequences of no group, beyond max_group_seqs, shorter than the shared rows (they keep what they have), shared rows
    beyond max_shared_len or negative, no shared row at all."""
    ptr, shared = [2, 6, 9], [300, 100]
    own = [40, 60, 5, 0, 7, 9, 100, 1, 50, 30, 0]
    pool = shared_pool(ptr, shared, own, 2, 16, seed=21)
    pool.lens[4] = 130   # shorter than its group's 300 rows
    q = queries(pool.rng, len(own), 8)
    ref = P.decode(pool, q)
    P.check(shared_decode(dp, pool, q, ptr, shared), ref)
    P.check(shared_decode(dp, pool, q, ptr, shared, most=2), ref)
    P.check(shared_decode(dp, pool, q, ptr, shared, longest=90), ref)
    P.check(shared_decode(dp, pool, q, ptr, shared, longest=0), ref)
    P.check(shared_decode(dp, pool, q, ptr, [-4, 100], longest=300), ref)
    # a group that ends behind the last sequence, one that begins before the first
    pool = shared_pool([0, 3, 9], [40, 100], own[:9], 2, 16, seed=25)
    q = queries(pool.rng, 9, 8)
    P.check(shared_decode(dp, pool, q, [-3, 3, 40], [40, 100], most=9), P.decode(pool, q))


def test_shared_prefix_of_very_many_groups_and_sequences(dp):
    """100 groups over 300 sequences, of which some share nothing; more groups than are dealt out."""
    rng = np.random.default_rng(26)
    ptr = np.concatenate([[0], np.sort(rng.integers(0, 301, 99)), [300]])
    shared = rng.integers(0, 200, 100)
    pool = shared_pool(ptr, shared, list(rng.integers(0, 50, 300)), 1, 16, seed=26, idle=set(rng.integers(0, 300, 20)))
    q = queries(pool.rng, 300, 2)
    P.check(shared_decode(dp, pool, q, ptr, shared), P.decode(pool, q))
    pool = shared_pool(np.arange(4201), [16] * 4200, [3] * 4200, 1, 16, seed=27)
    q = queries(pool.rng, 4200, 1)
    P.check(shared_decode(dp, pool, q, np.arange(4201), [16] * 4200), P.decode(pool, q))
    P.check(shared_decode(dp, pool, q, [0, 1, 4200], [16, 0]), P.decode(pool, q))


def test_shared_prefix_without_rows(dp):
    pool = shared_pool([0, 3], [50], [4, 4, 4], 1, 16, seed=22, idle={0, 1, 2})
    pool.table = np.full((3, 4), -1, dtype=np.int32)
    q = queries(pool.rng, 3, 4)
    P.check(shared_decode(dp, pool, q, [0, 3], [50], max_len=64), P.decode(pool, q))


def test_shared_prefix_leaves_out_pages_that_are_not_there(dp):
    for page in (4, 16, 64):
        pool = shared_pool([0, 20], [500], [40] * 20, 1, page, seed=23)
        pool.table[:, 1] = -1
        pool.table[:, 3] = pool.n_pages
        pool.table[5, -1] = 2 ** 31 - 1
        q = queries(pool.rng, 20, 4)
        P.check(shared_decode(dp, pool, q, [0, 20], [500]), P.decode(pool, q))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shared_prefix_keeps_what_is_not_finite_in_its_place(dp, dtype):
    """An infinite value in a shared row stays in its dimension; shared rows that score -inf have no weight; all of them."""
    for lo, hi in ((0, 0), (64, 200), (0, 300)):
        pool = shared_pool([0, 9], [300], [20] * 9, 1, 16, seed=24)
        pool.k = P.to_bf16_bits(np.where(np.isnan(P.wide(pool.k)), np.nan, 0.3 * P.wide(pool.k)))
        pool.k[np.isnan(P.wide(pool.k))] = P.NAN
        q = queries(pool.rng, 9, 4)
        q[..., 7] = H_ONE
        for r in range(lo, hi):
            pool.k[pool.table[0, r // 16], 0, r % 16, 7] = H_NINF
            for s in range(9):   # (the page in which the shared rows end is everybody's own)
                pool.k[pool.table[s, r // 16], 0, r % 16, 7] = H_NINF
        P.check(shared_decode(dp, pool, q, [0, 9], [300], dtype=dtype), P.decode(pool, q), dtype)
        if hi < 300:
            pool.v[pool.table[0, 250 // 16], 0, 250 % 16, 5] = H_INF
            out, _ = shared_decode(dp, pool, q, [0, 9], [300], dtype=dtype)
            assert torch.isposinf(out[..., 5]).all() and torch.isfinite(out).sum() == out.numel() - 9 * 4


@pytest.mark.parametrize("page", [4, 64])
def test_shared_groups_of_heads_side_by_side(dp, page):
    """Own rows of four KV heads per workgroup behind shared ones."""
    ptr, shared = [1, 6, 8], [333, 1000]
    pool = shared_pool(ptr, shared, [40, 200, 33, 0, 90, 7, 1500, 61, 300], 4, page, seed=52, idle=(3,))
    longest, width = wide_bound(9, 4, page)
    longest, width = max(longest + 1024, 2500), max(width + -(-1024 // page), -(-2500 // page))
    pool.table = np.pad(pool.table, ((0, 0), (0, width - pool.table.shape[1])), constant_values=-1)
    q = queries(pool.rng, 9, 20)
    P.check(shared_decode(dp, pool, q, ptr, shared, layout="token", max_len=longest), P.decode(pool, q))


@pytest.mark.parametrize("n_seqs", [9, 40])
def test_shared_rows_that_score_the_lowest_numbers(dp, n_seqs):
    for scores in (lambda i: np.full(len(i), LOWEST), lambda i: np.where(i < 64, LOWEST, -2.0 ** 127)):
        pool = shared_pool([0, n_seqs], [304], [20] * n_seqs, 1, 16, seed=42)
        q = queries(pool.rng, n_seqs, 4)
        only_dim_7(pool, q, scores)
        P.check(shared_decode(dp, pool, q, [0, n_seqs], [304], sm_scale=1.0), P.decode(pool, q, scale=1.0))


# ------------------------------------------------------------ used together --
def test_the_same_bits_twice(dp):
    pool = shared_pool([0, 30, 40], [2000, 700], list(range(40)), 2, 16, seed=31)
    q = queries(pool.rng, 40, 8)
    runs = [shared_decode(dp, pool, q, [0, 30, 40], [2000, 700]) for _ in range(2)]
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])
    runs = [paged(dp, pool, q) for _ in range(2)]
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])


def test_a_clustered_prompt_and_its_tail(dp):
    """The decode loop of a clustered cache: the step over the prompt's clusters (both thresholds at 1: every token), new
    tokens appended to pages at their positions in the whole context, their attention joined: dense attention over both."""
    from workloads import make_cache
    c = make_cache(batch=2, n_kv_heads=2, n_q_heads=8, context=[700, 300], mean_cluster=16, q_scale=0.4, seed=5)
    dc = dp.DeviceCache.from_host(c)
    pr = dp.Problem(dc)
    ws = torch.empty(dp.dp_workspace_bytes(pr), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(2, 8, 128, device="cuda"), torch.empty(2, 8, device="cuda")
    f = freqs_of(128)
    pool = P.Pool([0, 0], 2, 16, seed=32, width=4, spare=40)
    cache = pool.device(8, max_len=64)
    ws2 = torch.empty(dp.dp_paged_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    rng, base = pool.rng, np.array([700, 300])
    for step in range(20):
        cache.seq_lens += 1
        k, v = rng.standard_normal((2, 2, 2, 128))
        kd, vd = (torch.from_numpy(a).to(torch.bfloat16).cuda() for a in (k, v))
        pos = base + step
        dp.dp_append_kv(cache, kd, vd, torch.tensor(f, device="cuda"), positions=up(pos))
        for s in range(2):
            pool.put(s, step, P.rotate(P.wide(kd[s:s + 1]), pos[s:s + 1], f, False), P.wide(vd[s:s + 1]))
        pool.lens = np.array([step + 1] * 2, dtype=np.int32)
        dp.dp_decode_attention(pr, 1.0, 1.0, out, lse.view(-1), ws)
        dp.dp_paged_decode(cache, dc.q.view(torch.bfloat16), out, lse, ws2, prior_out=out, prior_lse=lse)
    torch.cuda.synchronize()
    # (what was appended may differ from the host's rounding by one step where the two angles straddle it)
    got = P.wide(cache.k_pages.view(torch.bfloat16)[up(pool.table[:, :2], np.int64)])
    assert np.abs(got - P.wide(pool.k[pool.table[:, :2]]))[np.isfinite(got)].max() <= 2 * P.BF16_HALF * 4
    pool.k = P.bits(cache.k_pages)
    import oracle
    ref, ref_lse, _ = oracle.Oracle(c).dense_step(n_threads=4)
    P.check((out, lse), P.decode(pool, c.q.reshape(2, 8, 128), prior=(ref, ref_lse)))


def serving_step(dp, cache, prefix, x, f, q_rot, out, lse, ws, n_kv=2):
    cache.seq_lens.add_(cache.seq_lens > 0)   # every live sequence grows by one token
    dp.dp_append_kv(cache, x[:, :n_kv], x[:, n_kv:2 * n_kv], f, q=x[:, 2 * n_kv:], q_out=q_rot)
    dp.dp_shared_prefix_decode(cache, prefix, q_rot, out[0], lse[0], ws[0])
    dp.dp_paged_decode(cache, q_rot, out[1], lse[1], ws[1])


def test_decode_steps_behind_a_shared_prompt_captured_and_replayed(dp):
    """A batch that grows token by token behind a shared prompt, an idle slot in it: append, shared and paged attention,
    eager, then captured once and replayed with other inputs and eager work in between; every step against 64 bits."""
    ptr, shared = [0, 5, 7], [200, 90]
    own = [3, 0, 15, 16, 30, 1, 60]
    pool = shared_pool(ptr, shared, own, 2, 16, seed=33, idle={1})
    need = -(-(pool.lens + 12) // 16)
    extra = P.Pool([0], 2, 16, seed=1, extra=20)   # (pages for what will be appended)
    pool.k, pool.v = np.concatenate([pool.k, extra.k]), np.concatenate([pool.v, extra.v])
    table = np.full((7, 20), -1, dtype=np.int32)
    table[:, :pool.table.shape[1]] = pool.table
    free = iter(range(pool.n_pages, pool.n_pages + 20))
    for s in range(7):
        for p in range(need[s]):
            if pool.lens[s] and table[s, p] < 0:
                table[s, p] = next(free)
    pool.table, pool.n_pages = table, pool.n_pages + 20
    cache = pool.device(8, max_len=320)
    prefix = dp.SharedPrefix(up(ptr), up(shared), 5, 200, dp.DP_SHARED_PREFIX_ONCE)
    f = freqs_of(128)
    fd = torch.tensor(f, device="cuda")
    x = torch.zeros(7, 12, 128, dtype=torch.bfloat16, device="cuda")
    q_rot = torch.empty(7, 8, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty(2, 7, 8, 128, device="cuda"), torch.empty(2, 7, 8, device="cuda")
    ws = [torch.full((n,), 255, dtype=torch.uint8, device="cuda")
          for n in (dp.dp_shared_prefix_workspace_bytes(cache, prefix), dp.dp_paged_workspace_bytes(cache))]
    gen = torch.Generator().manual_seed(5)

    def verify():
        torch.cuda.synchronize()
        pool.lens = cache.seq_lens.cpu().numpy()
        for s in range(7):
            if pool.lens[s]:
                pool.put(s, pool.lens[s] - 1, P.rotate(P.wide(x[s:s + 1, :2]), [pool.lens[s] - 1], f, False), P.wide(x[s:s + 1, 2:4]))
        pages = up(pool.table[pool.table >= 0], np.int64)
        got, want = P.wide(cache.k_pages.view(torch.bfloat16)[pages]), P.wide(pool.k[pool.table[pool.table >= 0]])
        assert np.array_equal(np.isnan(got), np.isnan(want))
        # one step of bf16 where the two sides' angles straddle a border, of values below 8
        assert np.nanmax(np.abs(got - want)) <= 2 * P.BF16_HALF * 8
        pool.k = P.bits(cache.k_pages).copy()
        ref = P.decode(pool, P.bits(q_rot))
        P.check((out[0], lse[0]), ref)
        P.check((out[1], lse[1]), ref)

    for _ in range(2):
        x.copy_(torch.randn(x.shape, generator=gen))
        serving_step(dp, cache, prefix, x, fd, q_rot, out, lse, ws)
        verify()
    graph = torch.cuda.CUDAGraph()
    lens = cache.seq_lens.clone()
    with torch.cuda.graph(graph):
        serving_step(dp, cache, prefix, x, fd, q_rot, out, lse, ws)
    cache.seq_lens.copy_(lens)
    for _ in range(4):
        x.copy_(torch.randn(x.shape, generator=gen))
        out.fill_(float("nan"))
        graph.replay()
        verify()
        torch.randn(1000, 1000, device="cuda").matmul(torch.randn(1000, 1000, device="cuda")).sum().item()
    x.copy_(torch.randn(x.shape, generator=gen))
    serving_step(dp, cache, prefix, x, fd, q_rot, out, lse, ws)
    verify()


def test_bound_calls_and_streams(dp):
    """Two bound calls with workspaces of their own on two streams at once, each against the plain call; a bound call
    follows the current stream unless it was given one."""
    pools = [P.Pool([3000, 50, 900], 2, 16, seed=s) for s in (41, 42)]
    qs = [queries(p.rng, 3, 8) for p in pools]
    refs = [P.decode(p, q) for p, q in zip(pools, qs)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    calls, outs = [], []
    for p, q in zip(pools, qs):
        c = p.device(8)
        o = torch.empty(3, 8, 128, device="cuda"), torch.empty(3, 8, device="cuda")
        ws = torch.full((dp.dp_paged_workspace_bytes(c),), 255, dtype=torch.uint8, device="cuda")
        outs.append(o)
        calls.append((dp.BoundCall(dp.dp_paged_decode, c, q_dev(q), *o, ws),
                      dp.BoundCall(dp.dp_paged_decode, c, q_dev(q), *o, ws, stream=streams[len(calls)])))
    torch.cuda.synchronize()
    for _ in range(5):
        for (current, fixed), s in zip(calls, streams):
            with torch.cuda.stream(s):
                current()
            fixed()
    torch.cuda.synchronize()
    for o, ref in zip(outs, refs):
        P.check(o, ref)
    # two captured graphs, each with its own buffers, replayed in turn and at once
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for (current, _), g in zip(calls, graphs):
        with torch.cuda.graph(g):
            current()
    for _ in range(3):
        for o, s, g in zip(outs, streams, graphs):
            with torch.cuda.stream(s):
                o[0].fill_(float("nan"))
                g.replay()
        torch.cuda.synchronize()
        for o, ref in zip(outs, refs):
            P.check(o, ref)
