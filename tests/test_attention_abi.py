"""Refusals of attention and of the quantised cache: every bad argument is turned away on the host, before any launch.
Needs no GPU."""
import ctypes
import math
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def A():
    if not os.path.exists(os.path.join(ROOT, "paper_2202_07471_amd", "libsquant_hip.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2202_07471_amd import attention
    attention._lib()
    return attention


P, WS, BIG = 0x10000, 0x20000, 1 << 40  # never dereferenced
NULL, SHAPE, MODE, WORKSPACE, FORMAT = 1, 2, 4, 5, 8
ref = ctypes.byref


def heads(A, data=P, row=512, head=64):
    return A.squant_heads_t(data, row, head)


def cache(A, kc=P, ks=P, vc=P, vs=P, pages=10, page=16, h=2, dim=64, fmt=1):
    return A.squant_cache_t(kc, ks, vc, vs, pages, page, h, dim, fmt)


def paged(A, table=P, lengths=P, starts=P, sequences=3, width=4):
    return A.squant_paged_t(table, lengths, starts, sequences, width)


def packed(A, qs=P, ks=P, sequences=3, q_rows=50, k_rows=60, h=4, kv=2, dim=64, causal=1, scale=0.5):
    return A.squant_packed_t(qs, ks, sequences, q_rows, k_rows, h, kv, dim, causal, scale)


BAD_CACHES = [(NULL, dict(kc=None)), (NULL, dict(ks=None)), (NULL, dict(vc=None)), (NULL, dict(vs=None)), (FORMAT, dict(fmt=2)),
              (FORMAT, dict(fmt=-1)), (FORMAT, dict(kc=P + 8)), (FORMAT, dict(vs=P + 1)), (SHAPE, dict(pages=0)), (SHAPE, dict(page=0)),
              (SHAPE, dict(h=0)), (SHAPE, dict(dim=48)), (SHAPE, dict(dim=0)), (SHAPE, dict(dim=512)), (SHAPE, dict(dim=-64)),
              (SHAPE, dict(pages=1 << 30, page=64))]
BAD_PLACES = [(SHAPE, dict(sequences=-1)), (SHAPE, dict(width=-1)), (NULL, dict(lengths=None)), (NULL, dict(table=None)),
              (FORMAT, dict(table=P + 2)), (FORMAT, dict(lengths=P + 1)), (FORMAT, dict(starts=P + 2)), (SHAPE, dict(starts=None))]
BAD_ROWS = [(NULL, dict(data=None)), (SHAPE, dict(row=63)), (SHAPE, dict(row=-512)), (SHAPE, dict(head=63)), (SHAPE, dict(row=1 << 41)),
            (SHAPE, dict(head=1 << 60))]


def test_rows_of_a_cache(A):
    L = A._lib()

    def write(k=None, v=None, type_=2, rows=5, c=None, w=None):
        return L.squant_cache_write(ref(k or heads(A)), ref(v or heads(A)), type_, rows, ref(c or cache(A)), ref(w or paged(A)), None)

    def read(k=None, v=None, type_=2, rows=5, c=None, w=None):
        return L.squant_cache_read(ref(c or cache(A)), ref(w or paged(A)), type_, rows, ref(k or heads(A)), ref(v or heads(A)), None)
    for f in (write, read):
        for want, bad in BAD_CACHES:
            assert f(c=cache(A, **bad)) == want, bad
        for want, bad in BAD_PLACES:
            assert f(w=paged(A, **bad)) == want, bad
        for want, bad in BAD_ROWS:
            assert f(k=heads(A, **bad)) == want and f(v=heads(A, **bad)) == want, bad
        assert f(type_=3) == FORMAT and f(type_=-1) == FORMAT and f(rows=-1) == SHAPE and f(rows=1 << 31) == SHAPE
        assert f(k=heads(A, data=P + 1)) == FORMAT and f(type_=0, v=heads(A, data=P + 2)) == FORMAT
        assert f(rows=0) == 0 and f(rows=0, w=paged(A, sequences=0, table=None, lengths=None)) == 0
    assert L.squant_cache_write(None, ref(heads(A)), 2, 5, ref(cache(A)), ref(paged(A)), None) == NULL
    assert L.squant_cache_write(ref(heads(A)), ref(heads(A)), 2, 5, None, ref(paged(A)), None) == NULL
    assert L.squant_cache_write(ref(heads(A)), ref(heads(A)), 2, 5, ref(cache(A)), None, None) == NULL


def test_attention_over_a_cache(A):
    L = A._lib()

    def f(q=None, type_=2, rows=5, h=8, c=None, w=None, scale=1.0, out=None, ws=WS, nbytes=BIG):
        return L.squant_cache_attention(ref(q or heads(A)), type_, rows, h, ref(c or cache(A)), ref(w or paged(A, width=400)), scale,
                                        ref(out or heads(A)), ws, nbytes, None)
    size = L.squant_cache_attention_workspace_bytes
    for want, bad in BAD_CACHES:
        assert f(c=cache(A, **bad)) == want and size(5, 8, ref(cache(A, **bad)), ref(paged(A))) == 0, bad
    for want, bad in BAD_PLACES:
        assert f(w=paged(A, **bad)) == want and size(5, 8, ref(cache(A)), ref(paged(A, **bad))) == 0, bad
    for want, bad in BAD_ROWS:
        assert f(q=heads(A, **bad)) == want and f(out=heads(A, **bad)) == want, bad
    assert f(h=7) == SHAPE and f(h=0) == SHAPE and f(h=-2) == SHAPE and f(type_=4) == FORMAT and f(rows=-1) == SHAPE
    assert f(scale=-1.0) == MODE and f(scale=math.nan) == MODE and f(scale=math.inf) == MODE
    assert f(ws=None) == WORKSPACE and f(nbytes=64) == WORKSPACE and f(ws=WS + 64) == WORKSPACE
    assert f(rows=1 << 30) == SHAPE and f(rows=0) == 0 and f(rows=0, ws=None, nbytes=0) == 0
    assert size(0, 8, ref(cache(A)), ref(paged(A))) == 0
    assert f(w=paged(A, width=(1 << 26) + 1)) == SHAPE and size(5, 8, ref(cache(A)), ref(paged(A, width=(1 << 26) + 1))) == 0
    # a table of a few hundred tokens needs none, a longer one does
    assert size(3, 8, ref(cache(A)), ref(paged(A, starts=None, width=8))) == 0
    one = size(3, 8, ref(cache(A)), ref(paged(A, starts=None, width=1000)))
    many = size(3000, 8, ref(cache(A)), ref(paged(A, starts=None, sequences=3000, width=1000)))
    assert 0 < one and many <= 1000 * one


def test_heads_of_a_cache(A):
    """What one call takes, all of them take."""
    L = A._lib()
    for h, dim, want in ((512, 256, 0), (513, 256, SHAPE), (4096, 32, 0), (4097, 32, SHAPE), (1 << 20, 64, SHAPE)):
        c, w, x = cache(A, h=h, dim=dim), paged(A, width=400), heads(A, row=1 << 18, head=dim)
        x.row = max(x.row, h * dim)
        none = paged(A, starts=P, width=400)
        assert L.squant_cache_write(ref(x), ref(x), 2, 0, ref(c), ref(none), None) == want
        assert L.squant_cache_read(ref(c), ref(none), 2, 0, ref(x), ref(x), None) == want
        assert L.squant_cache_attention(ref(x), 2, 0, h, ref(c), ref(w), 1.0, ref(x), WS, BIG, None) == want
        assert (L.squant_cache_attention_workspace_bytes(5, h, ref(c), ref(w)) > 0) == (want == 0)


def test_workspace_of_wide_tables(A):
    """What a table could hold does not decide how much memory a call takes."""
    size = A._lib().squant_cache_attention_workspace_bytes
    for rows in (1, 7, 96, 128, 1024, 20000):
        for h, kv, dim in ((1, 1, 32), (32, 8, 128), (64, 8, 128), (28, 4, 96), (16, 16, 256)):
            for tokens in (600, 16384, 131072, 1 << 20, 1 << 30):
                for starts, sequences in ((None, rows), (P, max(1, rows // 5))):
                    got = size(rows, h, ref(cache(A, h=kv, dim=dim)), ref(paged(A, starts=starts, sequences=sequences, width=tokens // 16)))
                    assert got <= (1 << 27) + 256, (rows, h, kv, dim, tokens)
                    if tokens >= 16384 and rows * h * dim <= 1 << 16:
                        assert got > 0  # few rows' long sequences are cut


def test_attention_over_prompts(A):
    L = A._lib()

    def f(q=None, k=None, v=None, type_=2, p=None, out=None, lse=P, ws=WS, nbytes=BIG):
        return L.squant_attention(ref(q or heads(A)), ref(k or heads(A)), ref(v or heads(A)), type_, ref(p or packed(A)), ref(out or heads(A)),
                                  lse, ws, nbytes, None)

    def g(d=None, q=None, k=None, v=None, out=None, lse=P, type_=2, p=None, dq=None, dk=None, dv=None, ws=WS, nbytes=BIG):
        return L.squant_attention_backward(*(ref(t or heads(A)) for t in (d, q, k, v, out)), lse, type_, ref(p or packed(A)),
                                           *(ref(t or heads(A)) for t in (dq, dk, dv)), ws, nbytes, None)
    for want, bad in [(SHAPE, dict(q_rows=-1)), (SHAPE, dict(k_rows=-1)), (SHAPE, dict(q_rows=1 << 31)), (SHAPE, dict(h=0)),
                      (SHAPE, dict(h=3)), (SHAPE, dict(kv=0)), (SHAPE, dict(dim=0)), (SHAPE, dict(dim=12)), (SHAPE, dict(dim=264)),
                      (SHAPE, dict(sequences=-1)), (NULL, dict(qs=None)), (NULL, dict(ks=None)), (SHAPE, dict(qs=None, ks=None)),
                      (FORMAT, dict(qs=P + 2)), (FORMAT, dict(ks=P + 1)), (MODE, dict(scale=-0.5)), (MODE, dict(scale=math.nan)),
                      (MODE, dict(scale=math.inf)), (MODE, dict(causal=2)), (SHAPE, dict(q_rows=1 << 30))]:
        assert f(p=packed(A, **bad)) == want and g(p=packed(A, **bad)) == want, bad
        assert L.squant_attention_backward_workspace_bytes(ref(packed(A, **bad)), 2) == 0
    for want, bad in BAD_ROWS:
        h = heads(A, **bad)
        assert all(f(**{x: h}) == want for x in ("q", "k", "v", "out")), bad
        assert all(g(**{x: h}) == want for x in ("d", "q", "k", "v", "out", "dq", "dk", "dv")), bad
    assert f(type_=3) == FORMAT and g(type_=-1) == FORMAT and f(lse=P + 2) == FORMAT and g(lse=P + 2) == FORMAT and g(lse=None) == NULL
    assert g(ws=None) == WORKSPACE and g(nbytes=8) == WORKSPACE and g(ws=WS + 16) == WORKSPACE
    assert f(p=packed(A, q_rows=0)) == 0 and g(p=packed(A, q_rows=0, k_rows=0), ws=None, nbytes=0) == 0
    alone = packed(A, sequences=1, q_rows=50, k_rows=2000)  # few rows and many keys are cut
    assert f(p=alone, ws=None) == WORKSPACE and f(p=alone, nbytes=100) == WORKSPACE and f(p=alone, ws=WS + 8) == WORKSPACE
    assert L.squant_attention_workspace_bytes(ref(alone), 2) > 2 * 50 * 4 * 64 * 4 and L.squant_attention_workspace_bytes(ref(alone), 7) == 0
    need = L.squant_attention_backward_workspace_bytes(ref(packed(A)), 2)
    assert need >= 50 * 4 * 4 and L.squant_attention_backward_workspace_bytes(ref(packed(A)), 3) == 0
    few, many = (L.squant_attention_backward_workspace_bytes(ref(packed(A, sequences=1, q_rows=n, k_rows=n)), 0) for n in (500, 50000))
    assert few > 500 * 4 * 4 * 64 and many == 50000 * 4 * 4  # a short sequence's walks are cut, a long one's are not


def test_the_binding_refuses(A):
    import paper_2202_07471_amd as sq
    q = torch.zeros(4, 2, 32)
    with pytest.raises(ValueError):
        sq.squant_attention(q, q, q)  # host tensors
    with pytest.raises(ValueError):
        sq.packed_attention(q, q, q)
    c = sq.QuantizedCache.empty(2, 2, 16, 32, device="cpu")
    assert c.key_codes.shape == (2, 2, 16, 16) and c.value_scales.shape == (2, 2, 16, 1)
    ints = torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        sq.squant_cache_write(q, q, c, ints, ints[:, 0])
    with pytest.raises(ValueError):
        sq.squant_cache_read(c, ints, ints[:, 0], None, 4, torch.float32)
    with pytest.raises(ValueError):
        sq.squant_cache_attention(q, c, ints, ints[:, 0])


def test_disjoint(A):
    """Never calls two places apart that share an element; knows slices of rows and of heads to be."""
    import random
    rng = random.Random(1)

    def place(h, shape):
        return {h.data // 2 + r * h.row + i * h.head + e for r in range(shape[0]) for i in range(shape[1]) for e in range(shape[2])}
    apart = 0
    for _ in range(4000):
        shapes = [(rng.randint(0, 4), rng.randint(0, 4), 4) for _ in range(2)]
        steps = [(rng.choice((4, 8, 12, 16, 20)), rng.choice((4, 8, 12, 16, 20))) for _ in range(2)]
        if rng.random() < 0.5:
            steps[1] = steps[0]
        hs = [A.squant_heads_t(64 + 2 * rng.randint(0, 40), *s) for s in steps]
        if A._disjoint(hs[0], shapes[0], hs[1], shapes[1], 2):
            assert not place(hs[0], shapes[0]) & place(hs[1], shapes[1])
            apart += 1
    assert apart > 1000
    fused = [A.squant_heads_t(64 + 2 * 4 * i, 32, 4) for i in (0, 4, 6)]
    shapes = [(9, 4, 4), (9, 2, 4), (9, 2, 4)]
    for i in range(3):
        for j in range(3):
            assert A._disjoint(fused[i], shapes[i], fused[j], shapes[j], 2) == (i != j)
