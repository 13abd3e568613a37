"""Attention over whole prompts and its gradients on the GPU, against their definitions in 64 bits."""
import math

import pytest
import torch

from attention_reference import BF16, F16, F32, attention64, close, packed64, starts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2202_07471_amd as sq
    sq.binding.lib()
    return sq


def inputs(seed, rows, keys, heads, kv, dim, dtype, peak=2.0):
    gen = torch.Generator().manual_seed(seed)
    q = (torch.randn(rows, heads, dim, generator=gen) * peak * torch.rand(rows, 1, 1, generator=gen)).to(dtype)
    k, v = (torch.randn(keys, kv, dim, generator=gen).to(dtype) for _ in range(2))
    dout = (torch.randn(rows, heads, dim, generator=gen) * 0.1).to(dtype)
    return q, k, v, dout


def both(sq, q, k, v, dout, qs, ks, scale, causal):
    q, k, v, dout = (t.cuda() for t in (q, k, v, dout))
    qs, ks = (None if s is None else s.cuda() for s in (qs, ks))
    out, lse = sq.squant_attention(q, k, v, qs, ks, scale, causal)
    return (out, lse) + sq.squant_attention_backward(dout, q, k, v, out, lse, qs, ks, scale, causal)


def check(sq, seed, q_counts, k_counts, heads, kv, dim, dtype, causal, q_pad=0, k_pad=0, scale=None):
    q, k, v, dout = inputs(seed, sum(q_counts) + q_pad, sum(k_counts) + k_pad, heads, kv, dim, dtype)
    scale = dim ** -0.5 if scale is None else scale
    got = both(sq, q, k, v, dout, starts_of(q_counts), starts_of(k_counts), scale, causal)
    r = packed64(q.double(), k.double(), v.double(), q_counts, k_counts, scale, causal, dtype, dout.double())
    for t, name in zip(got, ("out", "lse", "dq", "dk", "dv")):
        close(t, r, name, f"{q_counts} {k_counts} {heads}/{kv} x {dim} {dtype} {causal}")


LENGTHS = [([1], [1]), ([5], [5]), ([16], [33]), ([64], [64]), ([65], [127]), ([129], [129]), ([200, 1, 0, 77], [200, 1, 0, 77]),
           ([3, 130, 31], [40, 130, 95]), ([1, 1, 1], [300, 1, 64]), ([0, 0], [0, 0])]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("q_counts,k_counts", LENGTHS)
def test_lengths(sq, q_counts, k_counts, dtype, causal):
    check(sq, 1, q_counts, k_counts, 4, 2, 64, dtype, causal)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("dim", [8, 16, 32, 40, 64, 72, 80, 96, 104, 128, 136, 160, 192, 200, 224, 256])
def test_head_sizes(sq, dim, dtype):
    check(sq, dim, [70, 21], [70, 50], 2, 1, dim, dtype, True)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (7, 1), (6, 2), (12, 4), (8, 8)])
def test_heads(sq, heads, kv, dtype):
    check(sq, heads, [90, 45], [90, 45], heads, kv, 32, dtype, True)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_long(sq, dtype):
    check(sq, 3, [700, 333], [700, 1000], 2, 1, 128, dtype, True)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("causal", [True, False])
def test_few_rows_and_many_keys(sq, dtype, causal):
    """Walks that are cut: pieces that no row of a tile sees, rows that see nothing in some pieces."""
    check(sq, 18, [40], [2000], 2, 1, 64, dtype, causal)
    check(sq, 19, [5, 0, 130], [900, 1300, 60], 3, 1, 72, dtype, causal, q_pad=2, k_pad=1)
    check(sq, 20, [900], [20], 2, 2, 64, dtype, causal)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_that_see_nothing(sq, dtype, causal):
    """More queries than keys (causal: the first rows see none), a sequence without keys, one without queries, padding rows."""
    check(sq, 4, [40, 9, 0, 5], [17, 0, 12, 5], 4, 2, 64, dtype, causal, q_pad=7, k_pad=70)


@pytest.mark.parametrize("scale", [0.0, 1e-3, 1.0])
def test_scales(sq, scale):
    check(sq, 5, [50], [50], 2, 2, 64, BF16, True, scale=scale)


def test_one_sequence_without_starts(sq):
    q, k, v, dout = inputs(6, 100, 100, 2, 1, 64, BF16)
    r = packed64(q.double(), k.double(), v.double(), [100], [100], 0.125, True, BF16, dout.double())
    for t, name in zip(both(sq, q, k, v, dout, None, None, 0.125, True), ("out", "lse", "dq", "dk", "dv")):
        close(t, r, name)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_hidden_values(sq, dtype):
    """NaN and infinities in keys and values that a row does not see leave its output alone."""
    q, k, v, _ = inputs(7, 150, 150, 2, 1, 64, dtype)
    k2, v2 = k.clone(), v.clone()
    for at, value in ((60, math.nan), (101, math.inf), (149, -math.inf)):
        k2[at], v2[at] = value, value
    starts = starts_of([150]).cuda()
    one = sq.squant_attention(q.cuda(), k.cuda(), v.cuda(), starts)[0]
    two = sq.squant_attention(q.cuda(), k2.cuda(), v2.cuda(), starts)[0]
    r = attention64(q.double(), k.double(), v.double(), 0.125, True, dtype)
    r = {x: t[:60] for x, t in r.items()}
    close(one[:60], r, "out")
    close(two[:60], r, "out")
    assert two[60:].isnan().any(-1).all()
    # a padding key's contents, and those of the next sequence
    starts = starts_of([60, 41]).cuda()
    three = sq.squant_attention(q.cuda(), k2.cuda(), v2.cuda(), starts)[0]
    close(three[:60], r, "out")
    assert (three[101:] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_values_hidden_one_by_one(sq, dtype):
    """A value that is an infinity, its key ordinary: rows from it on are infinite there, rows before it are not touched."""
    q, k, v, _ = inputs(8, 70, 70, 1, 1, 64, dtype)
    v2 = v.clone()
    v2[33, 0, 5] = math.inf
    out = sq.squant_attention(q.cuda(), k.cuda(), v2.cuda())[0].cpu()
    want = sq.squant_attention(q.cuda(), k.cuda(), v.cuda())[0].cpu()
    assert (out[33:, 0, 5] == math.inf).all()
    v2[33, 0, 5] = 0
    r = attention64(q.double(), k.double(), v.double(), 0.125, True, dtype)
    r = {x: t[:33] for x, t in r.items()}
    close(out[:33], r, "out")
    close(want[:33], r, "out")


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_strides(sq, dtype):
    """Slices of one projection, an odd distance between rows, heads outside rows, results in given buffers."""
    heads, kv, dim, rows = 4, 2, 64, 75
    gen = torch.Generator().manual_seed(9)
    fused = torch.randn(rows, (heads + 2 * kv) * dim + 3, generator=gen).to(dtype).cuda()
    x = fused[:, 1:1 + (heads + 2 * kv) * dim].unflatten(1, (-1, dim))
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    dout = torch.randn(heads, rows, dim, generator=gen).to(dtype).cuda().transpose(0, 1)
    starts = starts_of([70, 5]).cuda()
    buf = torch.full((rows, heads * dim + 5), math.nan, dtype=dtype, device="cuda")
    out = buf[:, 2:2 + heads * dim].unflatten(1, (heads, dim))
    got, lse = sq.squant_attention(q, k, v, starts, out=out)
    assert got.data_ptr() == out.data_ptr()
    grads = torch.full((3, heads, rows, dim), math.nan, dtype=dtype, device="cuda")
    dq, dk, dv = grads[0].transpose(0, 1), grads[1, :kv].transpose(0, 1), grads[2, :kv].transpose(0, 1)
    sq.squant_attention_backward(dout, q, k, v, out, lse, starts, dq=dq, dk=dk, dv=dv)
    r = packed64(*(t.double().cpu() for t in (q, k, v)), [70, 5], [70, 5], dim ** -0.5, True, dtype, dout.double().cpu())
    for t, name in ((out, "out"), (lse, "lse"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        close(t, r, name)
    assert buf[:, :2].isnan().all() and buf[:, 2 + heads * dim:].isnan().all() and grads[1:, kv:].isnan().all()


def test_small_gradients_of_binary16(sq):
    """Gradients far below binary16's least normal number times a weight: still told apart."""
    q, k, v, dout = inputs(10, 200, 200, 2, 1, 64, F16)
    dout = (dout.float() * 2.0 ** -8).half()
    dout[:100] *= 2.0 ** -4
    r = packed64(q.double(), k.double(), v.double(), [100, 100], [100, 100], 0.125, False, F16, dout.double())
    got = both(sq, q, k, v, dout, starts_of([100, 100]), starts_of([100, 100]), 0.125, False)
    for t, name in zip(got, ("out", "lse", "dq", "dk", "dv")):
        close(t, r, name)


def test_autograd_and_differences(sq):
    """packed_attention's gradients: the definition's, through views and with some inputs that need none, and differences of the
    output along a direction."""
    q, k, v, w = (t.cuda() for t in inputs(11, 60, 60, 4, 2, 32, F32, peak=1.0))
    starts = starts_of([40, 20]).cuda()
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    out = sq.packed_attention(*leaves, starts)
    (out * w).sum().backward()
    r = packed64(*(t.double().cpu() for t in (q, k, v)), [40, 20], [40, 20], 32 ** -0.5, True, F32, w.double().cpu())
    for t, name in zip(leaves, ("dq", "dk", "dv")):
        close(t.grad, r, name)
    gen = torch.Generator(device="cuda").manual_seed(12)
    for leaf, at in zip(leaves, range(3)):
        d = torch.randn(leaf.shape, device="cuda", generator=gen)
        step = 2.0 ** -6
        ends = []
        for sign in (1, -1):
            x = [q, k, v]
            x[at] = x[at] + sign * step * d
            ends.append((sq.packed_attention(*x, starts).double() * w.double()).sum())
        slope = ((ends[0] - ends[1]) / (2 * step)).item()
        want = (leaf.grad.double() * d.double()).sum().item()
        # the step's square times a third derivative of order |d|^3 / sqrt(D)^3 per row, and rounding of 7680 terms over the step
        assert abs(slope - want) <= 0.01 * (leaf.grad.double().norm() * d.double().norm()).item() / 8
    k2 = k.clone().requires_grad_()
    sq.packed_attention(q, k2, v, starts).sum().backward()
    assert k2.grad.shape == k2.shape
    expanded = leaves[0].detach().clone().requires_grad_()
    sq.packed_attention(expanded, k, v, starts).sum().backward()  # the output's gradient is an expanded 1
    assert expanded.grad.isfinite().all()


def test_shared_heads_add_up(sq):
    """The gradient of a key head that query heads share is the sum of its copies' gradients."""
    q, k, v, dout = inputs(13, 64, 64, 6, 2, 64, F32)
    shared = both(sq, q, k, v, dout, None, None, 0.125, True)
    apart = both(sq, q, k.repeat_interleave(3, 1), v.repeat_interleave(3, 1), dout, None, None, 0.125, True)
    r = packed64(q.double(), k.double(), v.double(), [64], [64], 0.125, True, F32, dout.double())
    for i, name in ((3, "dk"), (4, "dv")):
        close(shared[i], r, name)
        close(apart[i].unflatten(1, (2, 3)).sum(2), {name: r[name], name + "_tol": 2 * r[name + "_tol"]}, name)


def test_same_bits(sq):
    q, k, v, dout = inputs(14, 513, 513, 8, 2, 128, BF16)
    one, two = (both(sq, q, k, v, dout, None, None, None, True) for _ in range(2))
    assert all(torch.equal(a, b) for a, b in zip(one, two))


def test_empty(sq):
    q, k, v, dout = inputs(15, 0, 9, 2, 1, 64, BF16)
    out, lse, dq, dk, dv = both(sq, q, k, v, dout, starts_of([0]), starts_of([9]), None, True)
    assert out.shape == q.shape and lse.shape == (2, 0) and dq.shape == q.shape and (dk == 0).all() and (dv == 0).all()
    q, k, v, dout = inputs(15, 9, 0, 2, 1, 64, BF16)
    out, lse, dq, dk, dv = both(sq, q, k, v, dout, starts_of([9]), starts_of([0]), None, True)
    assert (out == 0).all() and (lse == -math.inf).all() and (dq == 0).all() and dk.shape == k.shape


def test_streams_and_graphs(sq):
    """On a stream of their own, and captured: a replay gives what a call gives, with other lengths too."""
    q, k, v, dout = (t.cuda() for t in inputs(16, 200, 200, 4, 2, 64, BF16))
    starts = starts_of([120, 80]).cuda()
    want = sq.squant_attention(q, k, v, starts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sq.squant_attention(q, k, v, starts, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

    def step():
        out, lse = sq.squant_attention(q, k, v, starts)
        return (out, lse) + sq.squant_attention_backward(dout, q, k, v, out, lse, starts)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for counts in ([120, 80], [1, 150], [0, 0], [200, 0]):
        starts.copy_(starts_of(counts))
        q.mul_(0.75)
        torch.cuda.synchronize()
        graph.replay()
        for a, b in zip(held, step()):
            assert torch.equal(a, b)


def test_refusals(sq):
    q, k, v, dout = (t.cuda() for t in inputs(17, 8, 8, 4, 2, 64, BF16))
    starts = starts_of([8]).cuda()
    out, lse = sq.squant_attention(q, k, v, starts)
    bad = [lambda: sq.squant_attention(q, k.half(), v, starts), lambda: sq.squant_attention(q, k, v[:4], starts),
           lambda: sq.squant_attention(q, k[:4], v[:4], starts), lambda: sq.squant_attention(q, k[:, :, :32], v, starts),
           lambda: sq.squant_attention(q[:, :3], k, v, starts), lambda: sq.squant_attention(q, k, v, starts.long()),
           lambda: sq.squant_attention(q, k, v, starts, k_starts=starts[:1]), lambda: sq.squant_attention(q, k, v, k_starts=starts),
           lambda: sq.squant_attention(q, k, v, starts.cpu()), lambda: sq.squant_attention(q, k.cpu(), v, starts),
           lambda: sq.squant_attention(q, k, v, starts, scale=-1.0), lambda: sq.squant_attention(q, k, v, starts, scale=math.nan),
           lambda: sq.squant_attention(q[:, :, :60], k[:, :, :60], v[:, :, :60], starts),
           lambda: sq.squant_attention(q.transpose(1, 2), k, v, starts), lambda: sq.squant_attention(q.double(), k, v, starts),
           lambda: sq.squant_attention(q[:, :, ::2], k[:, :, ::2], v[:, :, ::2], starts),
           lambda: sq.squant_attention(q, k, v, starts, out=out[:, :, :32]),
           lambda: sq.squant_attention(q, k, v, starts, out=out[:1].expand(8, 4, 64)),
           lambda: sq.squant_attention_backward(dout[:4], q, k, v, out, lse, starts),
           lambda: sq.squant_attention_backward(dout, q, k, v, out, lse.half(), starts),
           lambda: sq.squant_attention_backward(dout, q, k, v, out, lse[:2], starts),
           lambda: sq.squant_attention_backward(dout, q, k, v, out, lse, starts, dk=k[:4])]
    for f in bad:
        with pytest.raises(ValueError):
            f()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("sequences", [63, 64, 200])
def test_many_sequences(sq, sequences, dtype):
    counts = [(7 * i) % 23 for i in range(sequences)]
    keys = [(5 * i) % 19 + (90 if i % 50 == 49 else 0) for i in range(sequences)]
    check(sq, 30, counts, keys, 2, 1, 32, dtype, True, q_pad=3, k_pad=2)


def test_output_over_the_queries(sq):
    for rows, keys in ((150, 150), (20, 2000)):  # the second is cut
        q, k, v, _ = (t.cuda() for t in inputs(31, rows, keys, 4, 2, 64, BF16))
        want, lse = sq.squant_attention(q, k, v)
        got, lse2 = sq.squant_attention(q, k, v, out=q)
        assert got is q and torch.equal(q, want) and torch.equal(lse, lse2)


def test_overlaps(sq):
    """Results beside what is read, in one buffer, are taken; over it they are refused."""
    rows, dim = 40, 32
    gen = torch.Generator().manual_seed(32)
    fused = torch.randn(rows, 4 + 2 + 2, dim, generator=gen).to(BF16).cuda()
    both_ = torch.cat((fused, torch.zeros(rows, 12, dim, dtype=BF16, device="cuda")), 1)
    q, k, v = both_[:, :4], both_[:, 4:6], both_[:, 6:8]
    out, lse = sq.squant_attention(q, k, v, out=both_[:, 8:12])
    want, _ = sq.squant_attention(q.clone(), k.clone(), v.clone())
    assert torch.equal(out, want)
    dout = torch.randn(rows, 4, dim, generator=gen).to(BF16).cuda()
    grads = torch.empty(rows, 8, dim, dtype=BF16, device="cuda")
    dq, dk, dv = grads[:, :4], grads[:, 4:6], grads[:, 6:]
    got = sq.squant_attention_backward(dout, q, k, v, out, lse, dq=dq, dk=dk, dv=dv)
    fresh = sq.squant_attention_backward(dout, q, k, v, out, lse)
    assert all(torch.equal(a, b) for a, b in zip(got, fresh))
    heads_first = torch.empty(8, rows, dim, dtype=BF16, device="cuda").transpose(0, 1)
    got = sq.squant_attention_backward(dout, q, k, v, out, lse, dq=heads_first[:, :4], dk=heads_first[:, 4:6], dv=heads_first[:, 6:])
    assert all(torch.equal(a, b) for a, b in zip(got, fresh))
    before = both_.clone()
    over_lse = lse.view(torch.uint8).flatten().view(BF16)[:rows * 2 * dim].unflatten(0, (-1, 2, dim))
    bad = [lambda: sq.squant_attention(q, k, v, out=both_[:, 1:5]), lambda: sq.squant_attention(q, k, v, out=both_[:, 5:9]),
           lambda: sq.squant_attention(q[:20], k, v, k_starts=None, out=both_[10:30, :4]),
           lambda: sq.squant_attention(q, k, v, out=both_.flatten()[16:16 + rows * 4 * dim].unflatten(0, (rows, 4, dim))),
           lambda: sq.squant_attention_backward(dout, q, k, v, out, lse, dq=q), lambda: sq.squant_attention_backward(dout, q, k, v, out, lse, dq=dout),
           lambda: sq.squant_attention_backward(dout, q, k, v, out, lse, dq=out), lambda: sq.squant_attention_backward(dout, q, k, v, out, lse, dk=v),
           lambda: sq.squant_attention_backward(dout, q, k, v, out, lse, dk=dk, dv=dk),
           lambda: sq.squant_attention_backward(dout, q, k, v, out, lse, dq=dq, dv=grads[:, 3:5]),
           lambda: sq.squant_attention_backward(dout, q[:, :, :], k[:5], v[:5], out, lse, k_starts=None, starts=None, dk=over_lse[:5])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    assert torch.equal(both_, before)


def test_two_streams_at_once(sq):
    sides = [torch.cuda.Stream() for _ in range(2)]
    work = [tuple(t.cuda() for t in inputs(33 + i, 600, 600, 6, 2, 96, F32)) for i in range(2)]
    want = [both(sq, *w, None, None, None, True) for w in work]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, (q, k, v, dout) in enumerate(work):
            out, lse = sq.squant_attention(q, k, v, stream=sides[i])
            got[i].append((out, lse) + sq.squant_attention_backward(dout, q, k, v, out, lse, stream=sides[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


def test_broken_starts(sq):
    """Starts that fall, are negative or beyond the rows: what is computed is anything, in the buffers given."""
    rows, dim = 300, 64
    q, k, v, dout = (t.cuda() for t in inputs(35, rows, rows, 2, 1, dim, BF16))
    for broken in ([0, 200, 100, 300], [5, 5, -7, 90], [0, 10 ** 9, 20, 2 ** 31 - 1], [300, 200, 100, 0]):
        starts = torch.tensor(broken, dtype=torch.int32).cuda()
        bufs = [torch.full((rows + 2, h, dim), 7.0, dtype=BF16, device="cuda") for h in (2, 2, 1, 1)]
        out, dq, dk, dv = (b[1:-1] for b in bufs)
        lse = sq.squant_attention(q, k, v, starts, out=out)[1]
        sq.squant_attention_backward(dout, q, k, v, out, lse, starts, dq=dq, dk=dk, dv=dv)
        assert all((b[0] == 7).all() and (b[-1] == 7).all() for b in bufs)


def test_autograd_in_a_graph(sq):
    """A captured training step; while an eager graph of the same leaves lives, the capture's call is refused."""
    q, k, v, dout = (t.cuda() for t in inputs(36, 130, 130, 4, 2, 64, BF16))
    starts = starts_of([100, 30]).cuda()
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    eager = sq.packed_attention(*leaves, starts)
    graph = torch.cuda.CUDAGraph()
    scratch = torch.ones(4, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        scratch.mul_(2.0)
        with pytest.raises(RuntimeError):
            sq.packed_attention(*leaves, starts)
    del eager
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(sq.packed_attention(*leaves, starts), leaves, dout)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sq.packed_attention(*leaves, starts)
        grads = torch.autograd.grad(out, leaves, dout)
    held = out.detach()
    del out
    for counts in ([100, 30], [1, 129], [60, 20]):
        starts.copy_(starts_of(counts))
        torch.cuda.synchronize()
        graph.replay()
        want, lse = sq.squant_attention(q, k, v, starts)
        want = (want,) + sq.squant_attention_backward(dout, q, k, v, want, lse, starts)
        for a, b in zip((held,) + grads, want):
            assert torch.equal(a, b)


def test_autograd_of_views(sq):
    """One sequence without starts; keys of one head for several, broadcast; queries whose elements are not beside each other."""
    q, k, v, w = (t.cuda() for t in inputs(37, 50, 50, 4, 1, 32, F32, peak=1.0))
    base = q.transpose(1, 2).contiguous().requires_grad_()
    k2, v2 = k.clone().requires_grad_(), v.clone().requires_grad_()
    out = sq.packed_attention(base.transpose(1, 2), k2.expand(50, 2, 32), v2.expand(50, 2, 32))
    out.backward(w)
    r = packed64(*(t.double().cpu() for t in (q, k, v)), [50], [50], 32 ** -0.5, True, F32, w.double().cpu())
    close(out, r, "out")
    close(base.grad.transpose(1, 2), r, "dq")
    for t, name in ((k2, "dk"), (v2, "dv")):
        close(t.grad, {name: r[name], name + "_tol": 2 * r[name + "_tol"]}, name)


def test_two_steps_of_one_graph(sq):
    """The same keys twice in a graph: their gradients add up; a second backward pass over a kept graph gives the same again."""
    q, k, v, w = (t.cuda() for t in inputs(38, 40, 40, 2, 1, 64, BF16))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    out = sq.packed_attention(*leaves)
    once = torch.autograd.grad(out, leaves, w, retain_graph=True)
    again = torch.autograd.grad(out, leaves, w)
    assert all(torch.equal(a, b) for a, b in zip(once, again))
    both_ = sq.packed_attention(leaves[0], leaves[1], leaves[1])
    both_.backward(w)
    _, dk, dv = both(sq, q, k, k, w, None, None, None, True)[2:]
    assert torch.equal(leaves[1].grad, dk + dv)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
def test_more_tiles_than_run_at_once(sq, causal, dtype):
    """Tiles in the order of their walks: sequences without queries or keys, more queries than keys, padding, all alike, 61 to 63 of them."""
    for q_counts, k_counts, heads, kv in (([0, 300, 17, 130, 260, 1, 129, 3], [5, 300, 90, 130, 400, 64, 0, 1], 64, 32), ([128] * 6, [128] * 6, 64, 64),
                                          ([260] * 4, [200, 260, 200, 264], 64, 32), ([5, 200], [700, 30], 128, 64)):
        check(sq, 39, q_counts, k_counts, heads, kv, 32, dtype, causal, q_pad=140, k_pad=70)
    for sequences in (61, 62, 63):
        counts = [(7 * i) % 23 + (200 if i % 20 == 19 else 0) for i in range(sequences)]
        check(sq, 40, counts, counts[::-1], 16, 16, 32, dtype, causal, q_pad=1)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_rows(sq, dtype):
    """Rows as far apart as they may be, the last ones beyond 2^32 bytes; further is refused."""
    rows, heads, kv, dim, step = 600 if dtype == BF16 else 300, 4, 2, 64, 1 << 22
    q, k, v, dout = (t.cuda() for t in inputs(41, rows, rows, heads, kv, dim, dtype))
    wide = torch.empty(rows, step, dtype=dtype, device="cuda")
    x = wide[:, :(2 * heads + 2 * kv + 2 * heads + 2 * kv) * dim].unflatten(1, (-1, dim))
    parts = x.split([heads, kv, kv, heads, heads, heads, kv, kv], 1)
    for a, b in zip(parts, (q, k, v, dout)):
        a.copy_(b)
    starts = starts_of([rows - 50, 50]).cuda()
    want, lse = sq.squant_attention(q, k, v, starts)
    want_grads = sq.squant_attention_backward(dout, q, k, v, want, lse, starts)
    out, lse2 = sq.squant_attention(*parts[:3], starts, out=parts[4])
    grads = sq.squant_attention_backward(parts[3], *parts[:3], out, lse2, starts, dq=parts[5], dk=parts[6], dv=parts[7])
    for a, b in zip((out, lse2) + grads, (want, lse) + want_grads):
        assert torch.equal(a, b)
    cache = sq.QuantizedCache.empty(2, kv, rows, dim)
    args = (torch.tensor([[1]], dtype=torch.int32).cuda(), torch.tensor([rows], dtype=torch.int32).cuda(), starts_of([rows]).cuda())
    near = sq.QuantizedCache.empty(2, kv, rows, dim)
    sq.squant_cache_write(parts[1], parts[2], cache, *args)
    sq.squant_cache_write(k, v, near, *args)
    assert all(torch.equal(a[1].view(torch.int8), b[1].view(torch.int8)) for a, b in zip(cache, near))
    sq.squant_cache_read(cache, *args, rows, dtype, k=parts[6], v=parts[7])
    for a, b in zip(parts[6:], sq.squant_cache_read(cache, *args, rows, dtype)):
        assert torch.equal(a, b)
    sq.squant_cache_attention(parts[0], cache, *args, out=parts[5])
    assert torch.equal(parts[5], sq.squant_cache_attention(q, cache, *args))
    del wide, x, parts, out, grads
    far = torch.empty(3 * (step + 8), dtype=dtype, device="cuda").view(3, -1)[:, :heads * dim].unflatten(1, (heads, dim))
    with pytest.raises(sq.SQuantError):
        sq.squant_attention(far, k[:3], v[:3])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [40, 64, 72, 96])
def test_many_heads(sq, dim, dtype):
    """Gradients by 32 rows a wave."""
    check(sq, 42, [300, 200, 65], [280, 200, 90], 160, 80, dim, dtype, True, q_pad=3)
    check(sq, 43, [130, 257], [257, 140], 288, 144, dim, dtype, False, k_pad=5)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype,power", [(BF16, 24), (BF16, 60), (F16, 24), (F32, 24), (F32, 60)])
@pytest.mark.parametrize("rows,keys", [(100, 100), (3, 900)])
def test_scores_of_any_size(sq, rows, keys, dtype, power, sign):
    """Scores so far apart that a row's output is the value of its largest one, where a product's rounding is more than a weight's exponent."""
    gen = torch.Generator().manual_seed(81)
    count = torch.randperm(keys, generator=gen) % 97 + 1  # scores are multiples of 2^power / 8; equal ones have equal values
    half = power // 2
    q = torch.zeros(rows, 2, 64)
    k, v = torch.zeros(keys, 1, 64), torch.randn(100, 1, 64, generator=gen)[count]
    q[..., 0], k[..., 0] = 2.0 ** (power - half + 2), sign * count[:, None].float() * 2.0 ** (half - 3)
    q, k, v = (t.to(dtype) for t in (q, k, v))
    ints = dict(dtype=torch.int32, device="cuda")
    out, lse = sq.squant_attention(q.cuda(), k.cuda(), v.cuda(), torch.tensor([0, rows], **ints), torch.tensor([0, keys], **ints))
    score = sign * count.double() * 2.0 ** (power - 4)
    for i in range(rows):
        best = score[:keys - rows + i + 1].argmax()
        # equal scores' weights and their sum: rounded once each, to the element type and in binary32
        tol = (2.0 ** -20 + (2 if dtype != F32 else 0) * torch.finfo(dtype).eps / 2 + torch.finfo(dtype).eps / 2) * v[best].double().abs()
        assert ((out[i].cpu().double() - v[best].double()).abs() <= tol).all(), i
        want = score[best] + (score[:keys - rows + i + 1] == score[best]).double().sum().log()
        assert ((lse[:, i].cpu().double() - want).abs() <= 2.0 ** -21 * want.abs()).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,keys", [(40, 160), (3, 900), (300, 300)])
def test_large_values(sq, rows, keys, dtype):
    """Values whose sums leave binary32 where weights are more than 1, and stay within it where they are not."""
    gen = torch.Generator().manual_seed(84)
    q, k = torch.zeros(rows, 2, 64), torch.zeros(keys, 1, 64)
    q[..., 0] = 8.0
    k[..., 0] = torch.arange(keys)[:, None] // 32 * 0.75  # largest scores that rise by little with each tile
    v = (1 + torch.rand(keys, 1, 64, generator=gen)) * 2.0 ** 120
    q, k, v = (t.to(dtype) for t in (q, k, v))
    ints = dict(dtype=torch.int32, device="cuda")
    out, lse = sq.squant_attention(q.cuda(), k.cuda(), v.cuda(), torch.tensor([0, rows], **ints), torch.tensor([0, keys], **ints))
    ref = attention64(q.double(), k.double(), v.double(), 0.125, True, dtype)
    close(out, ref, "out")
    close(lse, ref, "lse")
