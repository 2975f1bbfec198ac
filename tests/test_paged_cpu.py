"""Refusals of the entry points over a paged cache, and the reference that their tests use (CPU; nothing is launched)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2602_05191_amd as dp
from paper_2602_05191_amd import binding as B

import paged as P

INVALID, UNSUPPORTED, SMALL = -1, -2, -3
ONE = 256   # a pointer that nothing follows


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(dp.library_path()):
        from paper_2602_05191_amd import build
        build.build()
    return dp.load_library()


def cache(**kw):
    base = dict(n_seqs=4, n_kv_heads=2, n_q_heads=8, head_dim=128, n_pages=100, page_size=16, page_stride=2 * 16 * 128,
                head_stride=16 * 128, slot_stride=128, k_pages=ONE, v_pages=ONE, page_table=ONE, table_stride=10,
                max_seq_len=160, seq_lens=ONE, sm_scale=0.0)
    base.update(kw)
    return B._PagedCache(**base)


def append(**kw):
    base = dict(n_tokens=4, dtype=0, q=ONE, k=ONE, v=ONE, q_out=ONE, q_stride=1024, k_stride=256, v_stride=256,
                tok_ptr=None, positions=None, rope_freqs=ONE, rope_dims=128, flags=0)
    base.update(kw)
    return B._KvAppend(**base)


def prefix(**kw):
    base = dict(n_groups=1, max_group_seqs=4, max_shared_len=64, group_ptr=ONE, shared_lens=ONE, flags=0)
    base.update(kw)
    return B._SharedPrefix(**base)


BAD_CACHES = [
    (INVALID, dict(n_seqs=0)), (INVALID, dict(n_q_heads=7)), (INVALID, dict(n_kv_heads=0)), (INVALID, dict(n_pages=-1)),
    (INVALID, dict(page_size=0)), (INVALID, dict(slot_stride=132)), (INVALID, dict(head_stride=-8)),
    (INVALID, dict(page_stride=12)), (INVALID, dict(max_seq_len=161)), (INVALID, dict(max_seq_len=-1)),
    (INVALID, dict(table_stride=-1)), (INVALID, dict(k_pages=None)), (INVALID, dict(v_pages=None)),
    (INVALID, dict(k_pages=264)), (INVALID, dict(page_table=None)), (INVALID, dict(seq_lens=None)),
    (INVALID, dict(sm_scale=-1.0)), (INVALID, dict(sm_scale=float("nan"))),
    (UNSUPPORTED, dict(head_dim=64)), (UNSUPPORTED, dict(page_size=24)), (UNSUPPORTED, dict(page_size=48)),
    (UNSUPPORTED, dict(n_seqs=1 << 22)), (UNSUPPORTED, dict(n_seqs=(1 << 31) - 1)),
    (UNSUPPORTED, dict(slot_stride=1 << 30)), (UNSUPPORTED, dict(slot_stride=1 << 62)),
    (UNSUPPORTED, dict(max_seq_len=(1 << 30) + 1, table_stride=1 << 27)),
    (UNSUPPORTED, dict(n_seqs=1 << 14, max_seq_len=1 << 22, table_stride=1 << 18)),
    (UNSUPPORTED, dict(page_stride=1 << 60)), (UNSUPPORTED, dict(head_stride=1 << 60)),
]


@pytest.mark.parametrize("status, bad", BAD_CACHES)
def test_caches_that_are_refused(lib, status, bad):
    c, a, p, one = cache(**bad), append(), prefix(), C.c_void_p(ONE)
    assert lib.dp_append_kv(C.byref(c), C.byref(a), None) == status
    assert lib.dp_paged_decode(C.byref(c), one, None, None, None, one, 1, None, one, 1 << 40, None) == status
    assert lib.dp_shared_prefix_decode(C.byref(c), C.byref(p), one, one, 1, None, one, 1 << 40, None) == status
    assert lib.dp_paged_workspace_bytes(C.byref(c)) == 0
    assert lib.dp_shared_prefix_workspace_bytes(C.byref(c), C.byref(p)) == 0


@pytest.mark.parametrize("status, bad", [
    (INVALID, dict(n_tokens=-1)), (INVALID, dict(n_tokens=5)), (INVALID, dict(k=None)), (INVALID, dict(v=None)),
    (INVALID, dict(q_out=None)), (INVALID, dict(rope_freqs=None)), (INVALID, dict(flags=2)), (INVALID, dict(k=264)),
    (INVALID, dict(q=264)), (INVALID, dict(q_out=260)), (INVALID, dict(v_stride=-256)), (INVALID, dict(k_stride=260)),
    (INVALID, dict(q_stride=1 << 60)),
    (UNSUPPORTED, dict(n_tokens=(1 << 25) + 1, tok_ptr=ONE)), (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(rope_dims=8)), (UNSUPPORTED, dict(rope_dims=144)),
    (UNSUPPORTED, dict(rope_dims=-16)),
])
def test_appends_that_are_refused(lib, status, bad):
    assert lib.dp_append_kv(C.byref(cache()), C.byref(append(**bad)), None) == status
    assert lib.dp_append_kv(C.byref(cache()), None, None) == INVALID


def test_an_append_of_nothing_is_no_error(lib):
    assert lib.dp_append_kv(C.byref(cache()), C.byref(append(n_tokens=0, k=None, v=None, tok_ptr=ONE)), None) == 0


def test_decodes_that_are_refused(lib):
    c, one = C.byref(cache()), C.c_void_p(ONE)
    call = lambda q=one, first=None, po=None, pl=None, out=one, dt=1, ws=one, n=1 << 40: lib.dp_paged_decode(  # noqa: E731
        c, q, first, po, pl, out, dt, None, ws, n, None)
    assert call(q=None) == INVALID and call(q=C.c_void_p(264)) == INVALID and call(out=None) == INVALID
    assert call(po=one) == INVALID and call(pl=one) == INVALID and call(ws=None) == INVALID
    assert call(ws=C.c_void_p(128)) == INVALID and call(dt=2) == UNSUPPORTED
    assert call(n=lib.dp_paged_workspace_bytes(c) - 1) == SMALL


def test_a_prior_of_fp32_is_not_joined_in_place_of_bf16(lib):
    c, one, other = C.byref(cache()), C.c_void_p(ONE), C.c_void_p(2 * ONE)
    call = lambda out, dt: lib.dp_paged_decode(c, one, None, other, other, out, dt, None, one, 0, None)  # noqa: E731
    bf16, fp32 = 0, 1
    assert call(other, bf16) == INVALID and call(one, bf16) == SMALL and call(other, fp32) == SMALL


@pytest.mark.parametrize("bad", [dict(n_groups=0), dict(max_group_seqs=0), dict(max_shared_len=-1),
                                 dict(max_shared_len=161), dict(group_ptr=None), dict(shared_lens=None), dict(flags=2)])
def test_shared_prefixes_that_are_refused(lib, bad):
    c, p, one = C.byref(cache()), prefix(**bad), C.c_void_p(ONE)
    assert lib.dp_shared_prefix_decode(c, C.byref(p), one, one, 1, None, one, 1 << 40, None) == INVALID
    assert lib.dp_shared_prefix_workspace_bytes(c, C.byref(p)) == 0
    good = C.byref(prefix())
    assert lib.dp_shared_prefix_decode(c, good, one, one, 1, None, one,
                                       lib.dp_shared_prefix_workspace_bytes(c, good) - 1, None) == SMALL
    assert lib.dp_shared_prefix_decode(c, None, one, one, 1, None, one, 1 << 40, None) == INVALID


def host_cache(**kw):
    n = dict(k=torch.zeros(6, 2, 16, 128, dtype=torch.bfloat16), table=torch.zeros(3, 2, dtype=torch.int32),
             lens=torch.zeros(3, dtype=torch.int32), longest=32, heads=4)
    n.update(kw)
    return dp.PagedCache(n["k"], n.get("v", n["k"]), n["table"], n["lens"], n["longest"], n["heads"])


@pytest.mark.parametrize("bad", [
    dict(k=torch.zeros(6, 2, 16, 128)), dict(v=torch.zeros(6, 2, 8, 128, dtype=torch.bfloat16)),
    dict(k=torch.zeros(6, 2, 128, 16, dtype=torch.bfloat16).transpose(2, 3)), dict(lens=torch.zeros(3, dtype=torch.int64)),
    dict(lens=torch.zeros(2, dtype=torch.int32)), dict(table=torch.zeros(3, 2)), dict(longest=33),
    dict(table=torch.zeros(1, 2, dtype=torch.int32).expand(3, 2))])
def test_the_binding_refuses_caches(bad):
    host_cache()
    with pytest.raises(AssertionError):
        host_cache(**bad)


def test_the_binding_refuses_calls():
    c = host_cache()
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    k, f = bf(3, 2, 128), torch.ones(64)
    for kw in (dict(k=bf(2, 2, 128)), dict(v=k.float()), dict(k=bf(3, 128, 2).transpose(1, 2)), dict(q=bf(3, 4, 128)),
               dict(q=bf(3, 4, 128), q_out=torch.zeros(3, 4, 128)), dict(tok_ptr=torch.zeros(3, dtype=torch.int32)),
               dict(rope_freqs=f.double()), dict(positions=torch.zeros(2, dtype=torch.int32)), {}):   # (last: no GPU)
        with pytest.raises(AssertionError):
            dp.dp_append_kv(**dict(dict(cache=c, k=k, v=k, rope_freqs=f), **kw))
    q, out, ws = bf(3, 4, 128), torch.zeros(3, 4, 128), torch.zeros(256, dtype=torch.uint8)
    for kw in (dict(q=q.float()), dict(out=out[:2]), dict(lse=torch.zeros(3)), dict(prior_out=out),
               dict(first_rows=torch.zeros(3)), {}):
        with pytest.raises(AssertionError):
            dp.dp_paged_decode(**dict(dict(cache=c, q=q, out=out, lse=None, workspace=ws), **kw))
    with pytest.raises(AssertionError):
        dp.BoundCall(dp.dp_paged_decode, c, q, out, None, ws)
    with pytest.raises(AssertionError):
        dp.SharedPrefix(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 1, 1)


def test_the_reference_is_a_softmax():
    """The reference of the GPU tests against torch's softmax in 64 bits; a prior that is the rest of the rows."""
    pool = P.Pool([40, 0, 7], n_kv=2, page=8, seed=5)
    q = P.to_bf16_bits(pool.rng.standard_normal((3, 6, 128)))
    out, lse = P.decode(pool, q)
    k, v = pool.rows(0, 0, 40)
    x = torch.from_numpy(P.wide(q[0, 3:])) @ torch.from_numpy(k[1]).T / 128 ** 0.5
    assert np.abs((torch.softmax(x, 1) @ torch.from_numpy(v[1])).numpy() - out[0, 3:]).max() < 1e-12
    assert np.abs(torch.logsumexp(x, 1).numpy() - lse[0, 3:]).max() < 1e-12
    assert (out[1] == 0).all() and np.isneginf(lse[1]).all()
    lens, first = pool.lens, [25, 0, 3]
    pool.lens = np.asarray(first)
    head = P.decode(pool, q)
    pool.lens = lens
    both = P.decode(pool, q, first=first, prior=head)
    assert np.abs(both[0] - out).max() < 1e-12 and np.abs(both[1][[0, 2]] - lse[[0, 2]]).max() < 1e-12


def test_the_reference_turns_pairs():
    x = np.zeros((1, 1, 128))
    x[..., 0] = 1.0
    f = [np.pi / 2] + [0.0] * 15
    assert np.abs(P.rotate(x, [1], f, True)[0, 0, 1] - 1) < 1e-15 and np.abs(P.rotate(x, [1], f, False)[0, 0, 16] - 1) < 1e-15
    assert np.abs(P.rotate(x, [2], f, True)[0, 0, 0] + 1) < 1e-15


ROWS = 4 * 8 * 128   # elements of q_out: 4 tokens of 8 heads
FAR = 1 << 30


@pytest.mark.parametrize("bad", [
    dict(dtype=1),                                                    # fp32 queries in place: rows of q_out lie on other tokens'
    dict(q_stride=1536), dict(q_stride=0),                            # in place, not contiguous
    dict(q=FAR + 16), dict(q=FAR - 16), dict(q=FAR + 2 * ROWS - 16), dict(q=FAR - 2 * ROWS + 16),
    dict(q=FAR - 3 * 2 * 1536, q_stride=1536),                        # the last token's row is q_out's first
    dict(q=FAR - 2 * 2 * 99328 - 2 * 1008, q_stride=99328),           # one token's last 16 numbers reach it, q_out lies in a gap else
    dict(q=FAR + 2 * ROWS - 2 * 8, q_stride=99328),
    dict(k=FAR), dict(v=FAR), dict(k=FAR + 2 * ROWS - 16), dict(v=FAR - 3 * 512 - 512 + 16),
    dict(k=FAR - 2 * 2048, k_stride=1024), dict(v=FAR + 4096, v_stride=0),
    dict(n_tokens=1, tok_ptr=ONE, dtype=1),
])
def test_rotated_queries_that_would_overwrite_what_is_read(lib, bad):
    kw = dict(q=FAR, q_out=FAR, k=2 * FAR, v=3 * FAR)
    kw.update(bad)
    assert lib.dp_append_kv(C.byref(cache()), C.byref(append(**kw)), None) == INVALID


@pytest.mark.parametrize("heads, rows", [(200, 64 * 10737417), (256, 64 * ((1 << 23) - 3) + 1), (128, 64 * ((1 << 24) - 5)), (510, 64 * 4210751)])
def test_rows_are_counted_in_32_bits(lib, heads, rows):
    """A call's chunks of 64 rows, and one round of shares of them that 512 workgroups take, stay below 2^31: what passes it
    is refused, what is just below is not."""
    def room(rows):
        c = cache(n_seqs=1, n_kv_heads=heads, n_q_heads=heads, page_size=1 << 14, page_stride=0, head_stride=0, slot_stride=8,
                  max_seq_len=rows, table_stride=1 << 17)
        return lib.dp_paged_workspace_bytes(C.byref(c))
    while True:
        chunks = heads * -(-rows // 64)
        share = -(-chunks // 512)
        if 512 * share < 1 << 31 and chunks + 511 < 1 << 31:
            break
        assert room(rows) == 0
        rows -= 64
    assert room(rows - 2 * 64) > 0
