"""Cross entropy over a vocabulary of codes on the GPU, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from lin_reference import TINY, U, codes_of, pack, strided, sum_error

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def sq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2202_07471_amd as sq
    sq.binding.lib()
    return sq


def case(t, d, v, dtype, fmt, size=1.0):
    rng = np.random.default_rng([t, d, v])
    h = torch.from_numpy((rng.standard_normal((t, d)) * size * rng.uniform(0.1, 4, (t, 1))).astype(np.float32)).to(dtype)
    c = codes_of(rng, v, d, fmt, False)
    unit = (1.0 if fmt == "int4" else 1.0 / 16) / np.sqrt(18.0 * d)
    scales = torch.from_numpy((rng.uniform(0.3, 2.0, v) * unit).astype(np.float32))
    labels = torch.from_numpy(rng.integers(0, v, t))
    labels[rng.random(t) < 0.15] = -100
    dloss = torch.from_numpy(rng.uniform(-1, 2, t).astype(np.float32))
    return h, c, scales, labels, dloss


def definition(h, c, scales, labels, dloss):
    w = c.double() * scales.double()[:, None]
    logits = h.double() @ w.t()
    lse = torch.logsumexp(logits, 1)
    live = labels >= 0
    y = torch.where(live, labels, 0)
    loss = torch.where(live, lse - logits.gather(1, y[:, None])[:, 0], 0.0)
    p = torch.exp(logits - lse[:, None])
    g = torch.where(live, dloss.double(), 0.0)
    dh = (p @ w - w[y]) * g[:, None]
    return w, logits, lse, loss, p, y, g, dh


SIZES = [(1, 1, 1), (1, 64, 5), (2, 100, 64), (7, 256, 1001), (16, 65, 130), (50, 512, 3001), (64, 64, 64), (65, 64, 257),
         (130, 333, 2000), (300, 130, 10007)]


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("t,d,v", SIZES)
def test_against_64_bits(sq, t, d, v, dtype, fmt):
    h, c, scales, labels, dloss = case(t, d, v, dtype, fmt)
    w, logits, lse, loss, p, y, g, dh = definition(h, c, scales, labels, dloss)
    rms = ((h.double() ** 2) @ (w.t() ** 2)).sqrt()
    e = sum_error(rms, d) + 2.0 ** -22 * logits.abs()  # of a logit
    e_lse = (p * e).sum(1) + 2.0 ** -20 + 2.0 ** -22 * lse.abs()
    codes = (pack(c) if fmt == "int4" else c).cuda()
    for pad in (0, 3):
        hh = strided(h, pad, "cuda")
        got_loss, got_lse = sq.squant_cross_entropy(hh, codes, scales.cuda(), labels.cuda())
        assert got_loss.dtype == F32 and got_lse.dtype == F32
        assert ((got_lse.cpu().double() - lse).abs() <= e_lse).all()
        live = labels >= 0
        assert ((got_loss.cpu().double() - loss).abs() <= e_lse + e.gather(1, y[:, None])[:, 0] + 2.0 ** -24 * loss).all()
        assert (got_loss.cpu()[~live] == 0).all()
        got = sq.squant_cross_entropy_backward(hh, codes, scales.cuda(), labels.cuda(), got_lse, dloss.cuda())
        assert got.dtype == dtype
        # a probability is off by its logit's error, and rounds to 12 bits (22 for binary32) of itself or 2^-38 of
        # the largest one possible: random errors, their root-sum-square taken 6 times
        operand = 2.0 ** -22 if dtype == F32 else 2.0 ** -12
        pw = ((p ** 2) @ (w ** 2)).sqrt()
        tol = (p * (e + e_lse[:, None] + 2.0 ** -21)) @ w.abs() + 6 * operand * pw + sum_error(pw, v) + 2.0 ** -22 * w[y].abs()
        tol = tol + 2.0 ** -36 * v ** 0.5 * scales.double().max() * c.double().abs().max()
        tol = g.abs()[:, None] * tol + U[dtype] * dh.abs() + TINY[dtype]
        assert ((got.cpu().double() - dh).abs() <= tol).all()
        assert (got.cpu()[~live] == 0).all()


def test_every_label_ignored_and_other_ignore_index(sq):
    h, c, scales, labels, dloss = case(70, 64, 300, BF16, "int8")
    none = torch.full_like(labels, 7)
    loss, lse = sq.squant_cross_entropy(h.cuda(), c.cuda(), scales.cuda(), none.cuda(), ignore_index=7)
    assert not loss.any() and torch.isfinite(lse).all()
    dh = sq.squant_cross_entropy_backward(h.cuda(), c.cuda(), scales.cuda(), none.cuda(), lse, dloss.cuda(), ignore_index=7)
    assert not dh.any()


@pytest.mark.parametrize("t", [5, 80])
def test_labels_outside_the_vocabulary_are_nan(sq, t):
    h, c, scales, labels, dloss = case(t, 64, 300, F16, "int4")
    labels[0], labels[1], labels[2], labels[3] = 300, -1, 2 ** 40, -2 ** 40
    labels[4] = 299
    codes = pack(c).cuda()
    loss, lse = sq.squant_cross_entropy(h.cuda(), codes, scales.cuda(), labels.cuda())
    dh = sq.squant_cross_entropy_backward(h.cuda(), codes, scales.cuda(), labels.cuda(), lse, dloss.cuda())
    assert torch.isnan(loss[:4]).all() and torch.isfinite(loss[4:]).all()
    assert torch.isnan(dh[:4]).all() and torch.isfinite(dh[4:]).all()
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("t", [9, 100])
def test_peaked_and_far_logits(sq, t):
    """Logits of hundreds: one entry takes all, exponentials of the others leave binary32."""
    h, c, scales, labels, dloss = case(t, 128, 2049, F32, "int8", size=300.0)
    w, logits, lse, loss, p, y, g, dh = definition(h, c, scales, labels, dloss)
    got_loss, got_lse = sq.squant_cross_entropy(h.cuda(), c.cuda(), scales.cuda(), labels.cuda())
    rms = ((h.double() ** 2) @ (w.t() ** 2)).sqrt().amax(1)
    tol = 2 * sum_error(rms, 128) + 2.0 ** -20 * (logits.abs().amax(1) + 1)
    assert ((got_lse.cpu().double() - lse).abs() <= tol).all()
    assert ((got_loss.cpu().double() - loss).abs() <= 2 * tol).all()
    got = sq.squant_cross_entropy_backward(h.cuda(), c.cuda(), scales.cuda(), labels.cuda(), got_lse, dloss.cuda())
    assert torch.isfinite(got).all()
    bound = (g.abs() * (2 * tol + 2.0 ** -18))[:, None] * w.abs().max()
    assert ((got.cpu().double() - dh).abs() <= bound * 4).all()


def test_bad_row_stays_alone(sq):
    h, c, scales, labels, dloss = case(70, 64, 300, BF16, "int8")
    labels[:] = 3
    h[5, 1] = float("nan")
    loss, lse = sq.squant_cross_entropy(h.cuda(), c.cuda(), scales.cuda(), labels.cuda())
    dh = sq.squant_cross_entropy_backward(h.cuda(), c.cuda(), scales.cuda(), labels.cuda(), lse, dloss.cuda())
    rest = [i for i in range(70) if i != 5]
    assert torch.isnan(loss[5]) and torch.isfinite(loss[rest]).all()
    assert torch.isnan(dh[5]).all() and torch.isfinite(dh[rest]).all()


def test_gradient_against_differences(sq):
    h, c, scales, labels, _ = case(12, 80, 500, F32, "int8")
    c, scales, labels = c.cuda(), scales.cuda(), labels.cuda()
    x = h.cuda().requires_grad_()
    sq.quantized_cross_entropy(x, c, scales, labels).sum().backward()
    v = torch.from_numpy(np.random.default_rng(3).standard_normal(tuple(h.shape)).astype(np.float32)).cuda()
    step = 2.0 ** -6
    up, down = (sq.squant_cross_entropy(h.cuda() + s * v, c, scales, labels)[0].double().sum().item() for s in (step, -step))
    got = (x.grad.double() * v.double()).sum().item()
    # third derivatives of a log-sum-exp stay below 1 for steps of logits of about 1; roundings 2^-20 / step
    assert abs((up - down) / (2 * step) - got) <= 1e-2 * max(1.0, abs(got))


def test_pieces_of_the_vocabulary(sq):
    """More rows than one piece of probabilities holds: several pieces, a ragged last one."""
    t, d, v = 40000, 16, 4096 * 2 + 77
    rng = np.random.default_rng(29)
    h = torch.from_numpy(rng.standard_normal((t, d)).astype(np.float32)).to(BF16)
    c = codes_of(rng, v, d, "int8", False)
    scales = torch.from_numpy(rng.uniform(0.001, 0.004, v).astype(np.float32))
    labels = torch.from_numpy(rng.integers(0, v, t))
    hg, cg, sg, lg = h.cuda(), c.cuda(), scales.cuda(), labels.cuda()
    loss, lse = sq.squant_cross_entropy(hg, cg, sg, lg)
    dh = sq.squant_cross_entropy_backward(hg, cg, sg, lg, lse, torch.ones(t, device="cuda"))
    rows = torch.from_numpy(rng.integers(0, t, 50))
    w, logits, lse64, loss64, p, y, g, want = definition(h[rows], c, scales, labels[rows], torch.ones(50))
    assert ((loss.cpu().double()[rows] - loss64).abs() <= 2.0 ** -16).all()
    assert ((dh.cpu().double()[rows] - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * (p ** 2 @ w ** 2).sqrt() + 2.0 ** -20).all()


def test_zero_rows_streams_and_a_graph(sq):
    h, c, scales, labels, dloss = case(90, 70, 700, BF16, "int4")
    h, codes, scales, labels, dloss = h.cuda(), pack(c).cuda(), scales.cuda(), labels.cuda(), dloss.cuda()
    loss, lse = sq.squant_cross_entropy(h[:0], codes, scales, labels[:0])
    assert loss.shape == (0,) and sq.squant_cross_entropy_backward(h[:0], codes, scales, labels[:0], lse, dloss[:0]).shape == (0, 70)

    def step(stream=None):
        loss, lse = sq.squant_cross_entropy(h, codes, scales, labels, stream=stream)
        return loss, lse, sq.squant_cross_entropy_backward(h, codes, scales, labels, lse, dloss, stream=stream)

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        h.copy_(torch.randn_like(h))
        for o in out:
            o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(step(), out)), f"replay {i}"


def test_a_last_piece_shorter_than_the_slices(sq):
    """The gradient's contraction is cut into slices by a whole piece; a last piece of two steps leaves some of them empty."""
    t, d, v = 2100, 64, 63744 + 70  # a piece holds 2^27 probabilities in whole tiles of 256 entries: 63744 for 2100 rows
    assert (1 << 27) // t // 256 * 256 == 63744
    rng = np.random.default_rng(43)
    h = torch.from_numpy(rng.standard_normal((t, d)).astype(np.float32)).to(BF16)
    c = codes_of(rng, v, d, "int8", False)
    scales = torch.from_numpy(rng.uniform(0.001, 0.004, v).astype(np.float32))
    labels = torch.from_numpy(rng.integers(63700, v, t))
    hg, cg, sg, lg = h.cuda(), c.cuda(), scales.cuda(), labels.cuda()
    loss, lse = sq.squant_cross_entropy(hg, cg, sg, lg)
    dh = sq.squant_cross_entropy_backward(hg, cg, sg, lg, lse, torch.ones(t, device="cuda"))
    rows = torch.from_numpy(rng.integers(0, t, 40))
    w, logits, lse64, loss64, p, y, g, want = definition(h[rows], c, scales, labels[rows], torch.ones(40))
    assert ((loss.cpu().double()[rows] - loss64).abs() <= 2.0 ** -16).all()
    assert ((dh.cpu().double()[rows] - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * (p ** 2 @ w ** 2).sqrt() + 2.0 ** -20).all()
