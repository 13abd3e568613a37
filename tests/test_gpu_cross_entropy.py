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


def likely_label_case(t, d, v, dtype, first_label=0, seed=0):
    """Rows whose label is their likeliest entry, with losses from 1 to 1e-5: each is the label's codes made as long as it takes, and noise."""
    rng = np.random.default_rng([t, d, v, seed])
    c = codes_of(rng, v, d, "int8", False)
    scales = torch.from_numpy((rng.uniform(0.5, 2.0, v) / (64.0 * np.sqrt(d))).astype(np.float32))
    w = c.double() * scales.double()[:, None]
    labels = torch.from_numpy(rng.integers(first_label, v, t))
    noise = 0.3 * torch.from_numpy(rng.standard_normal((t, d)))
    wanted = 10.0 ** -torch.linspace(0, 5, t, dtype=torch.float64)
    low, high = torch.zeros(t, dtype=torch.float64), torch.full((t,), 400.0, dtype=torch.float64)
    to = w[labels] / w[labels].norm(dim=1, keepdim=True)
    for _ in range(40):
        middle = (low + high) / 2
        logits = (noise + middle[:, None] * to) @ w.t()
        loss = torch.logsumexp(logits, 1) - logits.gather(1, labels[:, None])[:, 0]
        low, high = torch.where(loss > wanted, middle, low), torch.where(loss > wanted, high, middle)
    h = (noise + high[:, None] * to).to(dtype)
    dloss = torch.from_numpy(rng.uniform(0.5, 2, t).astype(np.float32))
    return h, c, scales, labels, dloss


def likely_label_bound(h, c, scales, labels, dloss, dtype):
    """(dh in 64 bits, how far it may be off).  dh = g sum_{v != y} p_v (w_v - w_y): every term is relative to the entries beside the label."""
    w, logits, lse, loss, p, y, g, _ = definition(h, c, scales, labels, dloss)
    assert (loss[-1] < 3e-5) and (loss[0] > 0.3)
    others = p.scatter(1, y[:, None], 0.0)
    dh = (others @ w - others.sum(1)[:, None] * w[y]) * g[:, None]  # without the cancellation of 1 - p
    rms = ((h.double() ** 2) @ (w.t() ** 2)).sqrt()
    e = sum_error(rms, h.shape[1]) + 2.0 ** -22 * logits.abs()  # of a logit
    e_lse = (p * e).sum(1) + 2.0 ** -20 + 2.0 ** -22 * lse.abs()
    off = others * (e + e_lse[:, None] + 2.0 ** -20)  # of a probability
    pw = ((others ** 2) @ (w ** 2)).sqrt()
    # a product's operand rounds to 2^-11 of itself (two halves: 2^-22) or 2^-38 of the largest one possible: random errors
    # of at most that, so 4 times their root-sum-square is seven times the sum's deviation
    operand = 2.0 ** -22 if dtype == F32 else 2.0 ** -11
    least = 2.0 ** -38 * scales.double().max() * (c.double() ** 2).sum(0).sqrt()
    tol = off @ w.abs() + off.sum(1)[:, None] * w[y].abs() + 4 * operand * pw + 4 * least + sum_error(pw, c.shape[0])
    tol = tol + 2.0 ** -20 * others.sum(1)[:, None] * w[y].abs()
    return dh, g.abs()[:, None] * tol + U[dtype] * dh.abs() + TINY[dtype]


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("t,d,v", [(7, 256, 2000), (50, 130, 517), (130, 256, 2049), (300, 512, 5000)])
def test_gradient_where_the_label_is_likely(sq, t, d, v, dtype, fmt):
    h, c, scales, labels, dloss = likely_label_case(t, d, v, dtype)
    if fmt == "int4":  # the same weights to four bits, scaled up
        c, scales = torch.clamp(torch.round(c.float() / 18), -7, 7).to(torch.int8), scales * 18
    want, tol = likely_label_bound(h, c, scales, labels, dloss, dtype)
    codes = (pack(c) if fmt == "int4" else c).cuda()
    _, lse = sq.squant_cross_entropy(h.cuda(), codes, scales.cuda(), labels.cuda())
    got = sq.squant_cross_entropy_backward(h.cuda(), codes, scales.cuda(), labels.cuda(), lse, dloss.cuda())
    bad = (got.cpu().double() - want).abs() > tol
    assert not bad.any(), f"rows {bad.any(1).nonzero()[:, 0].tolist()}"


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("first_label", [0, 4096])
def test_gradient_where_the_label_is_likely_in_pieces(sq, dtype, first_label):
    """So many rows that the vocabulary is taken in pieces of 4096 entries; labels anywhere, and all in the last piece."""
    h, c, scales, labels, dloss = likely_label_case(60, 64, 4096 * 2 + 77, dtype, 2 * first_label, seed=1)
    want, tol = likely_label_bound(h, c, scales, labels, dloss, dtype)
    times = 560
    hg, lg, gg = h.repeat(times, 1).cuda(), labels.repeat(times).cuda(), dloss.repeat(times).cuda()
    _, lse = sq.squant_cross_entropy(hg, c.cuda(), scales.cuda(), lg)
    got = sq.squant_cross_entropy_backward(hg, c.cuda(), scales.cuda(), lg, lse, gg).cpu().double().view(times, 60, 64)
    assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("t,d,v", [(7, 256, 2000), (50, 130, 517), (130, 256, 2049), (300, 512, 5000)])
def test_losses_of_likely_labels(sq, t, d, v, dtype):
    h, c, scales, labels, dloss = likely_label_case(t, d, v, dtype)
    labels[t // 2:] = ((h.double() @ (c.double() * scales.double()[:, None]).t()).argmax(1))[t // 2:]
    w, logits, lse, loss, p, y, g, _ = definition(h, c, scales, labels, dloss)
    others = p.scatter(1, y[:, None], 0.0)
    loss = -torch.log1p(-others.sum(1))
    got, _ = sq.squant_cross_entropy(h.cuda(), c.cuda(), scales.cuda(), labels.cuda())
    got = got.cpu().double()
    assert (got >= 0).all(), f"{(got < 0).sum().item()} of {t}"
    # a logit's error counts with 1 - p; a sum of at most 30 terms in a row from 1 on is off by 2^-24 for each
    e = sum_error(((h.double() ** 2) @ (w.t() ** 2)).sqrt(), d) + 2.0 ** -22 * logits.abs()
    tol = (others * (e + e.gather(1, y[:, None]))).sum(1) + 30 * 2.0 ** -24 + 2.0 ** -21 * loss
    assert ((got - loss).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t", [20, 130])
def test_losses_of_certain_labels_are_not_below_zero(sq, t, dtype):
    """Rows so long that the label takes all: the loss is 0 or next to it, and on the right side."""
    h, c, scales, labels, _ = likely_label_case(t, 256, 2049, dtype)
    size = torch.linspace(1, 6, t)[:, None]
    h = (h.float() * size).to(dtype)
    labels = (h.double() @ (c.double() * scales.double()[:, None]).t()).argmax(1)
    loss, _ = sq.squant_cross_entropy(h.cuda(), c.cuda(), scales.cuda(), labels.cuda())
    assert (loss >= 0).all(), f"{(loss < 0).sum().item()} of {t}, least {loss.min().item()}"
