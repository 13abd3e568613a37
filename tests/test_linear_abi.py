"""Refusals of the operators on quantised layers: every bad argument is turned away on the host, before any launch.
Needs no GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    lib_path = os.path.join(ROOT, "paper_2202_07471_amd", "libsquant_hip.so")
    if not os.path.exists(lib_path):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2202_07471_amd import linear
    return linear._lib()


P, WS = 0x10000, 0x20000  # never dereferenced
BIG = 1 << 40


def codes(cout=8, cin=64, fmt=0, c=P, s=P):
    from paper_2202_07471_amd.linear import squant_codes_t
    return ctypes.byref(squant_codes_t(c, s, cout, cin, fmt))


def linear(L, x=P, ldx=64, type_=0, rows=100, w=None, bias=P, act=0, res=P, ldr=8, y=P, ldy=8, keep=0, kept=None, ks=None,
           ws=WS, nbytes=BIG):
    return L.squant_linear(x, ldx, type_, rows, codes() if w is None else w, bias, act, res, ldr, y, ldy, keep, kept, ks, ws,
                           nbytes, None)


NULL, SHAPE, MODE, WORKSPACE, FORMAT = 1, 2, 4, 5, 8


@pytest.mark.parametrize("want,bad", [
    (NULL, dict(x=None)), (NULL, dict(y=None)), (NULL, dict(keep=1, ks=P)), (NULL, dict(keep=1, kept=P)),
    (NULL, dict(keep=2)), (SHAPE, dict(ldx=63)), (SHAPE, dict(ldy=7)), (SHAPE, dict(ldr=7)), (SHAPE, dict(rows=-1)),
    (SHAPE, dict(rows=1 << 40)), (FORMAT, dict(type_=3)), (FORMAT, dict(type_=-1)), (FORMAT, dict(x=P + 2)),
    (FORMAT, dict(y=P + 1)), (FORMAT, dict(bias=P + 2)), (FORMAT, dict(res=P + 2)), (FORMAT, dict(keep=2, kept=P + 1)),
    (FORMAT, dict(keep=1, kept=P, ks=P + 2)), (FORMAT, dict(type_=1, x=P + 1)), (MODE, dict(act=4)), (MODE, dict(act=-1)),
    (MODE, dict(keep=3)), (MODE, dict(keep=-1)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(nbytes=16)),
    (WORKSPACE, dict(ws=WS + 128)),
])
def test_linear(L, want, bad):
    assert linear(L, **bad) == want


def test_codes(L):
    for want, bad in [(NULL, dict(c=None)), (NULL, dict(s=None)), (SHAPE, dict(cout=0)), (SHAPE, dict(cin=-3)),
                      (SHAPE, dict(cout=1 << 25)), (FORMAT, dict(fmt=2)), (FORMAT, dict(fmt=-1)), (FORMAT, dict(s=P + 2))]:
        w = codes(**bad)
        assert linear(L, w=w) == want
        assert L.squant_linear_backward(P, 8, 0, 4, w, 0, 0, None, None, P, 64, P, WS, BIG, None) == want
        assert L.squant_cross_entropy(P, 64, 0, 4, w, P, -100, P, P, WS, BIG, None) == want
        assert L.squant_cross_entropy_backward(P, 64, 0, 4, w, P, -100, P, P, P, 64, WS, BIG, None) == want
        assert L.squant_linear_workspace_bytes(P, 64, 0, 4, w, 0) == 0
        assert L.squant_linear_backward_workspace_bytes(0, 4, w) == 0
        assert L.squant_cross_entropy_workspace_bytes(P, 64, 0, 4, w) == 0
        assert L.squant_cross_entropy_backward_workspace_bytes(P, 64, 0, 4, w) == 0
    assert linear(L, w=ctypes.POINTER(type(codes()._obj))()) == NULL


def test_backward(L):
    def f(dy=P, lddy=8, type_=0, rows=4, act=2, keep=2, z=P, zs=None, dx=P, lddx=64, db=P, ws=WS, nbytes=BIG):
        return L.squant_linear_backward(dy, lddy, type_, rows, codes(), act, keep, z, zs, dx, lddx, db, ws, nbytes, None)
    for want, bad in [(NULL, dict(dy=None)), (NULL, dict(dx=None)), (NULL, dict(z=None)), (NULL, dict(keep=1)),
                      (SHAPE, dict(lddy=7)), (SHAPE, dict(lddx=63)), (SHAPE, dict(rows=-1)), (FORMAT, dict(type_=5)),
                      (FORMAT, dict(dy=P + 2)), (FORMAT, dict(dx=P + 2)), (FORMAT, dict(z=P + 2)), (FORMAT, dict(db=P + 2)),
                      (MODE, dict(act=0)), (MODE, dict(keep=0)), (MODE, dict(act=7)), (MODE, dict(keep=9)),
                      (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(nbytes=0)), (WORKSPACE, dict(ws=WS + 8))]:
        assert f(**bad) == want, bad
    assert f(rows=0, db=None) == 0


def test_cross_entropy(L):
    def f(h=P, ldh=64, type_=0, rows=100, labels=P, loss=P, lse=P, ws=WS, nbytes=BIG):
        return L.squant_cross_entropy(h, ldh, type_, rows, codes(), labels, -100, loss, lse, ws, nbytes, None)

    def g(h=P, ldh=64, type_=0, rows=4, labels=P, lse=P, dloss=P, dh=P, lddh=64, ws=WS, nbytes=BIG):
        return L.squant_cross_entropy_backward(h, ldh, type_, rows, codes(), labels, -100, lse, dloss, dh, lddh, ws, nbytes, None)
    both = [(NULL, dict(h=None)), (NULL, dict(labels=None)), (NULL, dict(lse=None)), (SHAPE, dict(ldh=63)),
            (SHAPE, dict(rows=-2)), (FORMAT, dict(type_=3)), (FORMAT, dict(h=P + 2)), (FORMAT, dict(labels=P + 4)),
            (FORMAT, dict(lse=P + 2)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(nbytes=100)), (WORKSPACE, dict(ws=WS + 64))]
    for want, bad in both + [(NULL, dict(loss=None)), (FORMAT, dict(loss=P + 1))]:
        assert f(**bad) == want, bad
    for want, bad in both + [(NULL, dict(dloss=None)), (NULL, dict(dh=None)), (SHAPE, dict(lddh=63)), (FORMAT, dict(dh=P + 2)),
                             (FORMAT, dict(dloss=P + 2))]:
        assert g(**bad) == want, bad
    assert f(rows=0) == 0 and g(rows=0) == 0 and f(rows=0, ws=None, nbytes=0) == 0


def test_workspaces_grow_with_the_rows(L):
    for type_ in (0, 1, 2):
        sizes = [L.squant_linear_backward_workspace_bytes(type_, m, codes(1000, 700)) for m in (1, 100, 10000)]
        assert 0 < sizes[0] < sizes[1] < sizes[2]
        # the pieces of the probabilities bound what a long batch needs beside its rows
        w = codes(65536, 64)
        assert L.squant_cross_entropy_backward_workspace_bytes(P, 64, type_, 16384, w) < 1 << 30
    assert L.squant_linear_workspace_bytes(P, 64, 0, 0, codes(), 0) == 0


def test_the_binding_refuses():
    import paper_2202_07471_amd as sq
    x, c, s = torch.zeros(4, 8), torch.zeros(3, 8, dtype=torch.int8), torch.ones(3)
    with pytest.raises(ValueError):
        sq.squant_linear(x, c, s)                                   # host tensors
    with pytest.raises(ValueError):
        sq.squant_cross_entropy(x, c, s, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        sq.squant_linear_backward(torch.zeros(4, 3), c, s, 8)
    with pytest.raises(ValueError):
        sq.squant_linear(torch.zeros(()), c, s)
    with pytest.raises(ValueError):
        sq.quantized_linear(x, c, s, act=sq.ACT_GELU, keep=sq.KEEP_NONE)


def test_header_compiles_as_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "squant.h"\n'
                   'int probe(void) { squant_codes_t w; (void)w; return (int)SQUANT_ACT_SILU + (int)SQUANT_KEEP_FULL; }\n')
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-fsyntax-only",
                           "-I", os.path.join(ROOT, "include"), str(src)])


def test_the_gradient_of_a_long_batch_needs_no_more_for_a_larger_vocabulary(L):
    """Several pieces of the vocabulary add to the same sums."""
    small, large = (L.squant_cross_entropy_backward_workspace_bytes(P, 4096, 2, 32768, codes(v, 4096)) for v in (1 << 15, 1 << 18))
    assert large <= small * 1.1 and large < 2 << 30


def test_more_threads_than_a_launch_has_are_refused(L):
    """A launch counts its threads in 32 bits: rows of which each takes a workgroup."""
    assert L.squant_cross_entropy(P, 64, 0, 1 << 25, codes(), P, -100, P, P, WS, BIG, None) == SHAPE


@pytest.mark.parametrize("off", [lambda: torch.no_grad(), lambda: torch.inference_mode()])
def test_nothing_is_kept_for_a_backward_pass_that_cannot_come(monkeypatch, off):
    """Without gradients a layer whose bias is trained keeps no pre-activation; with them it does."""
    from paper_2202_07471_amd import linear
    keeps = []

    def call(x, codes, scales, bias=None, act=0, residual=None, keep=None, out=None, stream=None):
        keeps.append(keep)
        y = torch.zeros(x.shape[0], codes.shape[0])
        return y, {linear.KEEP_NONE: None, linear.KEEP_FULL: y.clone(), linear.KEEP_INT8: (y.to(torch.int8), y[:, :1])}[keep]

    monkeypatch.setattr(linear, "squant_linear", call)
    x, c, s = torch.zeros(4, 8), torch.zeros(3, 8, dtype=torch.int8), torch.ones(3)
    bias = torch.nn.Parameter(torch.zeros(3))
    for keep in (linear.KEEP_INT8, linear.KEEP_FULL):
        with off():
            linear.quantized_linear(x, c, s, bias, linear.ACT_GELU, keep=keep)
        linear.quantized_linear(x, c, s, bias, linear.ACT_GELU, keep=keep)
        linear.quantized_linear(x, c, s, bias.detach(), linear.ACT_GELU, keep=keep)
    none = linear.KEEP_NONE
    assert keeps == [none, linear.KEEP_INT8, none, none, linear.KEEP_FULL, none]


@pytest.mark.parametrize("type_", [0, 1, 2])
def test_a_call_with_a_launch_too_large_is_refused_before_its_first(L, type_):
    """From 2^24 rows on the loss would need 2^32 threads; without a device a launch would say 6."""
    fits, over = (1 << 24) - 1, 1 << 24
    for rows in (over, 1 << 25, 1 << 26):
        assert L.squant_cross_entropy(P, 64, type_, rows, codes(), P, -100, P, P, WS, 1 << 60, None) == SHAPE
        assert L.squant_cross_entropy_workspace_bytes(P, 64, type_, rows, codes()) == 0
    assert L.squant_cross_entropy_workspace_bytes(P, 64, type_, fits, codes()) > 0
    if type_ == 0:  # binary32 rows are laid out by a workgroup each; 16-bit ones are read as they are
        assert linear(L, rows=over, nbytes=1 << 60) == SHAPE
        assert L.squant_linear_workspace_bytes(P, 64, 0, over, codes(), 0) == 0 < L.squant_linear_workspace_bytes(P, 64, 0, fits, codes(), 0)
    big = codes(1 << 22, 1 << 22)  # 2^26 rows: more tiles than a launch has
    assert linear(L, type_=type_, rows=1 << 26, w=big, ldx=1 << 22, ldr=1 << 22, ldy=1 << 22, nbytes=1 << 62) == SHAPE
    assert L.squant_linear_backward(P, 1 << 22, type_, 1 << 26, big, 0, 0, None, None, P, 1 << 22, P, WS, 1 << 62, None) == SHAPE
    assert L.squant_linear_backward_workspace_bytes(type_, 1 << 26, big) == 0
    assert L.squant_cross_entropy_backward(P, 1 << 22, type_, 1 << 26, big, P, -100, P, P, P, 1 << 22, WS, 1 << 62, None) == SHAPE
    assert L.squant_cross_entropy_backward_workspace_bytes(P, 1 << 22, type_, 1 << 26, big) == 0


@pytest.mark.parametrize("shape", [(0,), (4, 0), (2, 3, 0), (0, 3, 0)])
def test_rows_without_elements_are_refused(shape):
    from paper_2202_07471_amd import linear
    with pytest.raises(ValueError):
        linear._rows(torch.zeros(shape), 0, "x")
