"""The product with codes and its gradient on the GPU, against their definitions in 64 bits.

Integer rows, integer codes and scales that are powers of two make every product and sum exact, so those outputs
have to be the exact value rounded once, bit for bit; the others are held to derived bounds.
"""
import numpy as np
import pytest
import torch

from lin_reference import TINY, U, act64, codes_of, pack, slope64, strided, sum_error

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def sq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2202_07471_amd as sq
    sq.binding.lib()
    return sq


def on_gpu(codes, fmt):
    return (pack(codes) if fmt == "int4" else codes).cuda()


def bits(t):
    return t.contiguous().view(torch.int32 if t.dtype == F32 else torch.int16).cpu()


def assert_rounded(got, want, dtype, what):
    want = want.to(F32).to(dtype) if dtype != F32 else want.to(F32)  # the exact values here are binary32 numbers
    got = got.cpu()
    same = (bits(got) == bits(want)) | ((got == 0) & (want == 0))
    assert same.all(), f"{what}: {(~same).sum().item()} of {same.numel()} differ, first at {(~same).nonzero()[0].tolist()}"


SIZES = [(1, 1, 1), (1, 64, 16), (1, 4096, 100), (2, 3, 5), (3, 65, 17), (7, 1000, 33), (16, 128, 64), (17, 127, 65),
         (33, 64, 130), (48, 520, 257), (64, 63, 1), (65, 64, 256), (65, 1, 300), (100, 200, 3), (130, 321, 511),
         (257, 130, 258), (300, 1028, 1000), (513, 64, 64), (700, 999, 1283)]


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_exact_products(sq, m, k, n, dtype, fmt):
    rng = np.random.default_rng([m, k, n])
    x = torch.from_numpy(rng.integers(-4, 5, (m, k)).astype(np.float32))
    c = codes_of(rng, n, k, fmt)
    scales = torch.from_numpy(2.0 ** rng.integers(-9, -5, n).astype(np.float32))
    bias = torch.from_numpy(rng.integers(-3, 4, n).astype(np.float32))
    res = torch.from_numpy(rng.integers(-3, 4, (m, n)).astype(np.float32))
    want = (x.double() @ c.double().t()) * scales.double() + bias.double() + res.double()
    for pad in (0, 3, 8):
        y = sq.squant_linear(strided(x.to(dtype), pad, "cuda"), on_gpu(c, fmt), scales.cuda(), bias.to(dtype).cuda(),
                             sq.ACT_NONE, strided(res.to(dtype), pad, "cuda"))
        assert_rounded(y, want, dtype, f"pad {pad}")


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_exact_gradients(sq, m, k, n, dtype, fmt):
    rng = np.random.default_rng([n, k, m])
    dy = torch.from_numpy(rng.integers(-4, 5, (m, n)).astype(np.float32))
    c = codes_of(rng, n, k, fmt)
    scales = torch.from_numpy(2.0 ** rng.integers(-9, -5, n).astype(np.float32))
    want = (dy.double() * scales.double()) @ c.double()
    for pad in (0, 5):
        dx, dbias = sq.squant_linear_backward(strided(dy.to(dtype), pad, "cuda"), on_gpu(c, fmt), scales.cuda(), k)
        assert_rounded(dx, want, dtype, f"dx, pad {pad}")
        assert_rounded(dbias, dy.double().sum(0), dtype, f"dbias, pad {pad}")
        assert sq.squant_linear_backward(strided(dy.to(dtype), pad, "cuda"), on_gpu(c, fmt), scales.cuda(), k,
                                         bias=False)[1] is None


def real_case(rng, m, k, n, dtype, fmt):
    x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32)).to(dtype)
    c = codes_of(rng, n, k, fmt, False)
    unit = (1.0 if fmt == "int4" else 1.0 / 16) / np.sqrt(12.0 * k)
    scales = torch.from_numpy((rng.uniform(0.5, 2.0, n) * unit).astype(np.float32))
    bias = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(dtype)
    return x, c, scales, bias


REAL = [(1, 300, 200), (5, 4096, 130), (40, 700, 1000), (200, 1280, 1000), (333, 2503, 641)]


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("m,k,n", REAL)
def test_layer_against_64_bits(sq, m, k, n, act, dtype, fmt):
    rng = np.random.default_rng([m, n, k])
    x, c, scales, bias = real_case(rng, m, k, n, dtype, fmt)
    res = torch.from_numpy(rng.standard_normal((m, n)).astype(np.float32)).to(dtype)
    w = c.double() * scales.double()[:, None]
    z = x.double() @ w.t() + bias.double()
    want = act64(z, act) + res.double()
    rms = ((x.double() ** 2) @ (w.t() ** 2)).sqrt()
    # slopes stay below 1.13; the activations themselves come within 2^-20 of their argument
    tol = U[dtype] * want.abs() + 1.13 * sum_error(rms, k) + 2.0 ** -20 * (z.abs() + 1) + TINY[dtype]
    args = (x.cuda(), on_gpu(c, fmt), scales.cuda(), bias.cuda(), sq.ACTS[act], res.cuda())
    y = sq.squant_linear(*args)
    assert ((y.cpu().double() - want).abs() <= tol).all()
    for keep in ("int8", "full"):
        y2, kept = sq.squant_linear(*args, keep=sq.KEEPS[keep])
        assert ((y2.cpu().double() - want).abs() <= tol).all()
        if keep == "full":
            assert ((kept.cpu().double() - z).abs() <= U[dtype] * z.abs() + sum_error(rms, k) + 2.0 ** -22 * (z.abs() + 1)).all()
            continue
        q, s = kept[0].cpu().double(), kept[1].cpu().double()
        for g in range(-(-n // 64)):
            cols = slice(64 * g, 64 * g + 64)
            e = sum_error(rms[:, cols], k) + 2.0 ** -22 * (z[:, cols].abs() + 1)
            top = z[:, cols].abs().amax(1)
            assert ((s[:, g] * 127 - top).abs() <= e.amax(1) + 2.0 ** -22 * top).all()
            # half a step of the code, and what z may be off by
            assert ((q[:, cols] * s[:, g:g + 1] - z[:, cols]).abs() <= s[:, g:g + 1] * (0.5 + 2.0 ** -14) + e).all()


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("m,k,n", REAL)
def test_gradient_against_64_bits(sq, m, k, n, act, dtype, fmt):
    rng = np.random.default_rng([k, m, n])
    _, c, scales, _ = real_case(rng, m, k, n, dtype, fmt)
    # rows of very different sizes, as loss scaling leaves them
    dy = torch.from_numpy((rng.standard_normal((m, n)) * 10.0 ** rng.uniform(-4, 2, (m, 1))).astype(np.float32)).to(dtype)
    w = c.double() * scales.double()[:, None]
    full = torch.from_numpy((2 * rng.standard_normal((m, n))).astype(np.float32)).to(dtype)
    q = torch.from_numpy(rng.integers(-127, 128, (m, n)).astype(np.int8))
    s = torch.from_numpy(rng.uniform(0.01, 0.05, (m, -(-n // 64))).astype(np.float32))
    q64 = q.double() * s.double().repeat_interleave(64, 1)[:, :n]
    for z, kept in ((full.double(), full.cuda()), (q64, (q.cuda(), s.cuda()))):
        dz = dy.double() * slope64(z, act)
        dx, dbias = sq.squant_linear_backward(dy.cuda(), on_gpu(c, fmt), scales.cuda(), k, sq.ACTS[act], kept)
        want = dz @ w
        rms = ((dz ** 2) @ (w ** 2)).sqrt()
        # an element of dz * scale rounds to 12 bits (22 for binary32) relative to itself, or 2^-38 of the row's
        # largest: random errors, their root-sum-square taken 6 times
        operand = 2.0 ** -22 if dtype == F32 else 2.0 ** -12
        slope_error = 2.0 ** -19 * ((dy.double().abs()) @ w.abs())
        tol = (U[dtype] * want.abs() + sum_error(rms, n) + 6 * operand * rms + slope_error + TINY[dtype]
               + 2.0 ** -36 * n ** 0.5 * (dy.double() * scales.double()).abs().amax(1, keepdim=True) * c.double().abs().max())
        assert ((dx.cpu().double() - want).abs() <= tol).all()
        want_b = dz.sum(0)
        tol_b = (U[dtype] * want_b.abs() + 2.0 ** -19 * dy.double().abs().sum(0)
                 + sum_error((dz ** 2).sum(0).sqrt(), m) + TINY[dtype])
        assert ((dbias.cpu().double() - want_b).abs() <= tol_b).all()


def test_gradient_against_differences(sq):
    """dx and dbias predict what the layer does a step away (binary32, a central difference)."""
    rng = np.random.default_rng(5)
    m, k, n = 9, 70, 45
    x, c, scales, bias = real_case(rng, m, k, n, F32, "int8")
    c, scales = c.cuda(), scales.cuda()
    dy = torch.from_numpy(rng.standard_normal((m, n)).astype(np.float32)).cuda()
    for act in ("gelu", "silu"):
        xg, bg = x.cuda().requires_grad_(), bias.cuda().requires_grad_()
        y = sq.quantized_linear(xg, c, scales, bg, sq.ACTS[act], keep=sq.KEEP_FULL)
        (y * dy).sum().backward()
        for t, g in ((x, xg.grad), (bias, bg.grad)):
            v = torch.from_numpy(rng.standard_normal(tuple(t.shape)).astype(np.float32))
            h = 2.0 ** -6

            def at(step):
                moved = (t + step * v).cuda()
                xx, bb = (moved, bias.cuda()) if t is x else (x.cuda(), moved)
                return (sq.squant_linear(xx, c, scales, bb, sq.ACTS[act]).double() * dy.double()).sum().item()

            got = (g.double().cpu() * v.double()).sum().item()
            # third derivatives below 2: h^2 / 6 * |v's change of z|^3 ; roundings 2^-20 / h
            assert abs((at(h) - at(-h)) / (2 * h) - got) <= 2e-2 * max(1.0, abs(got))


def test_autograd_of_expanded_and_strided(sq):
    rng = np.random.default_rng(7)
    x, c, scales, bias = real_case(rng, 6, 96, 80, BF16, "int4")
    packed, scales = pack(c).cuda(), scales.cuda()
    x3 = x.cuda().view(2, 3, 96).requires_grad_()
    b = bias.cuda().requires_grad_()
    r = torch.zeros(2, 3, 80, dtype=BF16, device="cuda", requires_grad=True)
    y = sq.quantized_linear(x3, packed, scales, b, sq.ACT_SILU, r)
    y.sum().backward()  # an expanded gradient: strides of zero
    assert torch.equal(r.grad, torch.ones_like(r))
    dx, db = sq.squant_linear_backward(torch.ones(6, 80, dtype=BF16, device="cuda"), packed, scales, 96, sq.ACT_SILU,
                                       tuple(t.view(6, -1) for t in sq.squant_linear(
                                           x.cuda(), packed, scales, b.detach(), sq.ACT_SILU, keep=sq.KEEP_INT8)[1]))
    assert torch.equal(x3.grad.view(6, 96), dx) and torch.equal(b.grad, db)
    y = sq.quantized_linear(x.cuda().t().contiguous().t(), packed, scales)  # columns first
    assert torch.equal(y, sq.squant_linear(x.cuda(), packed, scales))


@pytest.mark.parametrize("m", [1, 70])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_one_bad_row_stays_alone(sq, m, dtype):
    """Infinities and NaN of a row reach that row's outputs only; the rest of the tile is untouched."""
    rng = np.random.default_rng(11)
    x, c, scales, bias = real_case(rng, m + 2, 130, 70, dtype, "int8")
    x[1, 5] = float("nan")
    x[2 % (m + 2), 7] = float("inf")
    clean = x.clone()
    clean[1] = 0
    clean[2 % (m + 2)] = 0
    y = sq.squant_linear(x.cuda(), c.cuda(), scales.cuda(), bias.cuda(), sq.ACT_GELU).cpu()
    ref = sq.squant_linear(clean.cuda(), c.cuda(), scales.cuda(), bias.cuda(), sq.ACT_GELU).cpu()
    assert torch.isnan(y[1]).all()
    rest = [i for i in range(m + 2) if i not in (1, 2 % (m + 2))]
    assert torch.equal(y[rest], ref[rest])
    assert not torch.isfinite(y[2 % (m + 2)][c[:, 7] > 0]).any()
    _, kept = sq.squant_linear(x.cuda(), c.cuda(), scales.cuda(), bias.cuda(), sq.ACT_GELU, keep=sq.KEEP_INT8)
    assert torch.isnan(kept[1][1]).all() and torch.isfinite(kept[1][rest]).all()
    dy = torch.ones(m + 2, 70, dtype=dtype)
    dy[1, 3] = float("nan")
    dx, _ = sq.squant_linear_backward(dy.cuda(), c.cuda(), scales.cuda(), 130)
    assert torch.isnan(dx[1]).all() and torch.isfinite(dx[[i for i in range(m + 2) if i != 1]]).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_subnormal_rows(sq, dtype):
    """16-bit subnormals multiply as what they are."""
    x = torch.zeros(3, 64, dtype=dtype)
    x[0, 0], x[1, 1] = TINY[dtype], 3 * TINY[dtype]
    c = torch.ones(20, 64, dtype=torch.int8)
    for m in (3, 80):
        xx = x.repeat(27, 1)[:m]
        y = sq.squant_linear(xx.cuda(), c.cuda(), torch.full((20,), 4.0, device="cuda"))
        want = (xx.double().sum(1) * 4)[:, None].expand(m, 20)
        assert torch.equal(y.cpu().double(), want)


def test_large_and_small_binary32_rows(sq):
    """The exponent of a row covers binary32's range."""
    rng = np.random.default_rng(13)
    base = torch.from_numpy(rng.standard_normal((6, 100)).astype(np.float32))
    size = torch.tensor([2.0 ** 120, 2.0 ** -120, 1.0, 2.0 ** -140, 0.0, 2.0 ** 60])[:, None]
    x = base * size
    c = codes_of(rng, 40, 100, "int8")
    scales = torch.full((40,), 2.0 ** -7)
    for rows in (6, 90):
        xx = x.repeat(15, 1)[:rows]
        want = xx.double() @ c.double().t() * 2.0 ** -7
        rms = ((xx.double() ** 2) @ (c.double().t() * 2.0 ** -7) ** 2).sqrt()
        y = sq.squant_linear(xx.cuda(), c.cuda(), scales.cuda()).cpu().double()
        assert ((y - want).abs() <= sum_error(rms, 100) + 2.0 ** -24 * want.abs() + 2.0 ** -145).all()


def test_zero_rows_and_in_place_residual(sq):
    rng = np.random.default_rng(17)
    x, c, scales, bias = real_case(rng, 20, 64, 96, BF16, "int8")
    c, scales, bias = c.cuda(), scales.cuda(), bias.cuda()
    y = sq.squant_linear(x[:0].cuda(), c, scales, bias)
    assert y.shape == (0, 96)
    dx, db = sq.squant_linear_backward(y, c, scales, 64)
    assert dx.shape == (0, 64) and torch.equal(db, torch.zeros_like(bias))
    r = torch.randn(20, 96, device="cuda").to(BF16)
    want = sq.squant_linear(x.cuda(), c, scales, bias, sq.ACT_SILU, r)
    assert sq.squant_linear(x.cuda(), c, scales, bias, sq.ACT_SILU, r, out=r) is r and torch.equal(r, want)
    one = sq.squant_linear(x[0].cuda(), c, scales, bias)
    assert one.shape == (96,) and torch.equal(one, sq.squant_linear(x[:1].cuda(), c, scales, bias)[0])


def test_results_do_not_depend_on_the_run_or_the_batch(sq):
    """The same bits from run to run; a convolution's 4-d codes are their unfolded rows."""
    rng = np.random.default_rng(19)
    x, c, scales, bias = real_case(rng, 300, 18 * 9, 90, F16, "int8")
    a = sq.squant_linear(x.cuda(), c.cuda(), scales.cuda(), bias.cuda(), sq.ACT_GELU)
    for _ in range(3):
        assert torch.equal(a, sq.squant_linear(x.cuda(), c.view(90, 18, 3, 3).cuda(), scales.cuda(), bias.cuda(), sq.ACT_GELU))
    dy = torch.randn(300, 90, device="cuda").half()
    d = sq.squant_linear_backward(dy, c.cuda(), scales.cuda(), 162)
    for _ in range(3):
        e = sq.squant_linear_backward(dy, c.cuda(), scales.cuda(), 162)
        assert torch.equal(d[0], e[0]) and torch.equal(d[1], e[1])


def test_another_stream_and_a_graph(sq):
    rng = np.random.default_rng(23)
    x, c, scales, bias = real_case(rng, 150, 515, 260, BF16, "int8")
    x, c, scales, bias = x.cuda(), c.cuda(), scales.cuda(), bias.cuda()
    dy = torch.randn(150, 260, device="cuda").to(BF16)

    def step(stream=None):
        y, kept = sq.squant_linear(x, c, scales, bias, sq.ACT_SILU, keep=sq.KEEP_INT8, stream=stream)
        return (y,) + sq.squant_linear_backward(dy, c, scales, 515, sq.ACT_SILU, kept, stream=stream)

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
        x.copy_(torch.randn_like(x))
        for o in out:
            o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(step(), out)), f"replay {i}"


def test_offsets_beyond_32_bits(sq):
    """A weight of more than 2^32 codes: the last rows are right, and so are the last rows of activations."""
    k, n = 65536, 65536 + 96
    codes = torch.zeros(n, k, dtype=torch.int8, device="cuda")
    codes[-3:, :] = 1
    codes[-1, -1] = 5
    scales = torch.ones(n, device="cuda")
    for m in (2, 66):
        x = torch.ones(m, k, dtype=BF16, device="cuda")
        y = sq.squant_linear(x, codes, scales)
        assert torch.equal(y[:, -1], torch.full((m,), float(k + 4), dtype=BF16, device="cuda"))
        assert torch.equal(y[:, -2], torch.full((m,), float(k), dtype=BF16, device="cuda"))
        assert not y[:, :-3].any()
    dy = torch.zeros(2, n, dtype=BF16, device="cuda")
    dy[:, -1] = 1
    dx, _ = sq.squant_linear_backward(dy, codes, scales, k)
    assert (dx[:, :-1] == 1).all() and (dx[:, -1] == 5).all()


def test_memory_belongs_to_the_given_stream(sq):
    """Outputs of a call on another stream do not take memory that the current stream has just let go of."""
    rng = np.random.default_rng(31)
    x, c, scales, _ = real_case(rng, 600, 512, 1024, BF16, "int8")
    x, c, scales = x.cuda(), c.cuda(), scales.cuda()
    want = sq.squant_linear(x, c, scales)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    freed = torch.empty(600, 1024, dtype=BF16, device="cuda")
    at = freed.data_ptr()
    del freed
    y = sq.squant_linear(x, c, scales, stream=side)
    side.synchronize()
    assert y.data_ptr() != at and torch.equal(y, want)
    again = torch.empty(600, 1024, dtype=BF16, device="cuda")
    assert again.data_ptr() == at


@pytest.mark.parametrize("m", [3, 70])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_far_apart(sq, m, dtype):
    """More than 2^22 elements between rows: rows are laid out before the product."""
    rng = np.random.default_rng(37)
    x, c, scales, _ = real_case(rng, m, 128, 70, dtype, "int8")
    wide = torch.empty(m, (1 << 22) + 64, dtype=dtype, device="cuda")
    wide[:, 8:136] = x.cuda()
    assert torch.equal(sq.squant_linear(wide[:, 8:136], c.cuda(), scales.cuda()), sq.squant_linear(x.cuda(), c.cuda(), scales.cuda()))


def test_codes_changed_before_the_backward_pass_are_noticed(sq):
    rng = np.random.default_rng(41)
    x, c, scales, _ = real_case(rng, 9, 64, 48, F32, "int8")
    x, c, scales = x.cuda().requires_grad_(), c.cuda(), scales.cuda()
    y = sq.quantized_linear(x, c, scales)
    c.zero_()
    with pytest.raises(RuntimeError):
        y.sum().backward()
    loss = sq.quantized_cross_entropy(x, c, scales, torch.zeros(9, dtype=torch.int64, device="cuda"))
    scales.mul_(2)
    with pytest.raises(RuntimeError):
        loss.sum().backward()


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("k", [512, 516, 545, 2048 + 64, 32, 128])
@pytest.mark.parametrize("m,n", [(4100, 4128), (1030, 4352), (520, 1008)])
def test_exact_products_of_every_tile(sq, m, n, k, dtype, fmt):
    """Long and short contractions, code rows that begin at multiples of 16 bytes, of 4, and anywhere, and codes of which
    the first begins off them; the layer and its gradient."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + k)
    x = torch.randint(-4, 5, (m, k), device="cuda", generator=gen).float()
    dy = torch.randint(-4, 5, (m, n), device="cuda", generator=gen).float()
    c = codes_of(np.random.default_rng([m, k, n]), n, k, fmt)
    packed = (pack(c) if fmt == "int4" else c).cuda()
    scales = 2.0 ** torch.randint(-9, -5, (n,), device="cuda", generator=gen).float()
    c64 = c.double().cuda()
    want = (x.double() @ c64.t()) * scales.double()
    want_dx = (dy.double() * scales.double()) @ c64
    x, dy = x.to(dtype), dy.to(dtype)
    for off in (0, 4, 1):
        buf = torch.zeros(packed.numel() + 16, dtype=packed.dtype, device="cuda")
        w = buf[off:off + packed.numel()].view(packed.shape)
        w.copy_(packed)
        assert_rounded(sq.squant_linear(x, w, scales), want.cpu(), dtype, f"codes {off} bytes on")
        assert_rounded(sq.squant_linear_backward(dy, w, scales, k, bias=False)[0], want_dx.cpu(), dtype, f"dx, codes {off} bytes on")


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m,k", [(2, 40001), (16, 4100), (40, 2050), (64, 1024)])
def test_few_long_rows_between_words(sq, m, k, dtype, fmt):
    """16-bit rows that begin off 32-bit words, and enough of them that they are laid out first."""
    rng = np.random.default_rng([m, k])
    x = torch.from_numpy(rng.integers(-2, 3, (m, k)).astype(np.float32))
    c = codes_of(rng, 150, k, fmt)
    scales = torch.full((150,), 2.0 ** -8)
    want = (x.double() @ c.double().t()) * 2.0 ** -8
    labels = torch.from_numpy(rng.integers(0, 150, m)).cuda()
    lse = None
    for pad, begin in ((0, 0), (1, 0), (3, 1), (2, 1), (8, 0)):
        buf = torch.full((m, k + pad), float("nan"), dtype=dtype, device="cuda")
        view = buf[:, begin:begin + k]
        view.copy_(x)
        assert_rounded(sq.squant_linear(view, on_gpu(c, fmt), scales.cuda()), want, dtype, f"pad {pad}, from {begin}")
        got = sq.squant_cross_entropy(view, on_gpu(c, fmt), scales.cuda() / 64, labels)[1]
        lse = got if lse is None else lse
        assert torch.equal(got, lse)


@pytest.mark.parametrize("m", [5, 80])
@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -122, 2.0 ** -126, 2.0 ** -140])
def test_kept_codes_of_groups_next_to_zero(sq, m, size):
    """A group's largest |z| may be so small that 127 / it is no binary32 number: the codes are still rounded quotients, zeros among them."""
    rng = np.random.default_rng(47)
    z = torch.from_numpy(rng.integers(-100, 101, (m, 192)))
    z[:, ::3] = 0
    z[:, 64:128] = 0  # a group of zeros
    z[:, 1], z[:, 130] = 101, -102
    x = torch.zeros(m, 192)
    x[:] = z.float()
    c = torch.eye(192, dtype=torch.int8)
    _, (q, s) = sq.squant_linear(x.cuda(), c.cuda(), torch.full((192,), size, device="cuda"), keep=sq.KEEP_INT8)
    for g, top in ((0, 101.0), (1, 0.0), (2, 102.0)):
        want = z[:, 64 * g:64 * g + 64].double() * (127 / top) if top else torch.zeros(m, 64)
        # 2^-22 of a quotient of at most 127, which no quotient here is nearer to a half than
        assert ((q.cpu()[:, 64 * g:64 * g + 64] - want).abs() <= 0.5 + 2.0 ** -14).all(), f"group {g}"
        unit = top * size / 127 if top else 1.0
        assert ((s[:, g].cpu().double() - unit).abs() <= 2.0 ** -23 * unit + 2.0 ** -150).all()


def test_an_output_over_what_is_read_is_refused(sq):
    """Workgroups write while others still read: only the residual may be written over, in its own layout."""
    rng = np.random.default_rng(53)
    x, c, scales, bias = real_case(rng, 200, 96, 96, BF16, "int8")
    x, c, scales = x.cuda(), c.cuda(), scales.cuda()
    kept = x.clone()
    with pytest.raises(ValueError):
        sq.squant_linear(x, c, scales, out=x)
    wide = torch.zeros(200, 128, dtype=BF16, device="cuda")
    with pytest.raises(ValueError):  # the residual's rows 96 apart, the output's 128, from the same element on
        sq.squant_linear(x, c, scales, residual=wide.view(-1)[:200 * 96].view(200, 96), out=wide[:, :96])
    torch.cuda.synchronize()
    assert torch.equal(x, kept) and not wide.any()
    assert torch.equal(sq.squant_linear(x, c, scales, residual=wide[:, :96], out=wide[:, :96]), sq.squant_linear(x, c, scales))


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [1, 17, 32, 64])
@pytest.mark.parametrize("n", [1030, 2051, 4102, 8197, 12290])
def test_exact_products_of_few_rows_at_every_width(sq, m, n, dtype, fmt):
    """Each number of columns a workgroup, next to where the plan goes from one to the next."""
    rng = np.random.default_rng([m, n])
    x = torch.from_numpy(rng.integers(-4, 5, (m, 258)).astype(np.float32))
    c = codes_of(rng, n, 258, fmt)
    scales = torch.from_numpy(2.0 ** rng.integers(-9, -5, n).astype(np.float32))
    want = (x.double() @ c.double().t()) * scales.double()
    assert_rounded(sq.squant_linear(x.to(dtype).cuda(), on_gpu(c, fmt), scales.cuda()), want, dtype, "y")
