"""The quantised cache on the GPU: what is written and read bit for bit, attention over it against its definition in 64 bits."""
import math

import pytest
import torch

from attention_reference import BF16, F16, F32, GROUP, attention64, close, pack4, quantise, starts_of, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2202_07471_amd as sq
    sq.binding.lib()
    return sq


# Weights are binary16 numbers (binary32: sums of two) times 2^14 of a row's largest: half of 2^-24 over 2^14.
FLOOR = 2.0 ** -39


def formats(sq, bits):
    return sq.OUT_INT4 if bits == 4 else sq.OUT_INT8


def layout(gen, lengths, page, spare=2, wider=0):
    """(number of pages, table [sequences, width]) with the pages of each sequence anywhere."""
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=gen).to(torch.int32)
    table = torch.full((len(lengths), max(need + [0]) + wider), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return pages, table


def slots_of(table, page, b, first, last):
    t = torch.arange(first, last)
    return table[b, t // page].long(), t % page


def filled(sq, gen, pages, heads, page, dim, bits):
    """A cache of random values, and the same on the host."""
    host = []
    for _ in range(2):
        c, s = quantise(torch.randn(pages, heads, page, dim, generator=gen) * torch.exp2(torch.randint(-4, 4, (pages, heads, page, 1), generator=gen)), bits)
        host += [pack4(c) if bits == 4 else c, s]
    return sq.QuantizedCache(*(t.cuda() for t in host)), host


CASES = [(4, 1, 16), (8, 2, 16), (4, 3, 24), (8, 1, 7), (4, 8, 1), (8, 2, 100), (4, 2, 64)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("bits,heads,page", CASES)
def test_write_and_read(sq, bits, heads, page, dim, dtype):
    gen = torch.Generator().manual_seed(dim + page)
    lengths, new = [33, 1, 70, 0, 12], [20, 1, 70, 0, 3]
    pages, table = layout(gen, lengths, page, wider=1)
    rows = sum(new) + 5  # padding behind
    x = torch.randn(rows, 2 * heads * dim + 3, generator=gen).to(dtype)
    fused = x.cuda()[:, 1:1 + 2 * heads * dim].unflatten(1, (2 * heads, dim))
    k, v = fused[:, :heads], fused[:, heads:]
    cache, host = filled(sq, gen, pages, heads, page, dim, bits)
    args = (table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts_of(new).cuda())
    sq.squant_cache_write(k, v, cache, *args)
    r = 0
    wide = [torch.zeros(rows, heads, dim, dtype=torch.float64) for _ in range(2)]
    for b, (n, m) in enumerate(zip(new, lengths)):
        p, s = slots_of(table, page, b, m - n, m)
        for i, t in enumerate((k, v)):
            c, sc = quantise(t[r:r + n].cpu(), bits)
            host[2 * i][p, :, s] = pack4(c) if bits == 4 else c
            host[2 * i + 1][p, :, s] = sc
            wide[i][r:r + n] = values(c, sc)
        r += n
    for got, want in zip(cache, host):
        assert torch.equal(got.cpu().view(torch.uint8 if got.element_size() == 1 else torch.int16),
                           want.view(torch.uint8 if want.element_size() == 1 else torch.int16))
    for got, want in zip(sq.squant_cache_read(cache, *args, rows, dtype), wide):
        assert torch.equal(got.cpu(), want.to(dtype))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_borders(sq, bits, dtype):
    """Values a code and a half from each other, zeros, numbers too small for a scale, infinities and NaN."""
    top = 7 if bits == 4 else 127
    x = torch.zeros(12, 1, 64)
    for r in range(6):
        unit = 2.0 ** (r - 3)
        x[r, 0, :32] = (torch.arange(32).float() - 16 + 0.5).clamp(-top, top) * unit
        x[r, 0, 31] = top * unit
        x[r, 0, 32:] = torch.arange(32).float() * 0.37 * unit
    x[6, 0, :32] = 2.0 ** -133  # the scale is below bfloat16's least number
    x[7, 0, 3] = 2.0 ** -120
    x[8, 0, 5], x[8, 0, 40] = math.nan, 1.0
    x[9, 0, 5], x[9, 0, 63] = math.inf, -math.inf
    x[10] = torch.linspace(-6e4, 6e4, 64)
    if dtype != F16:
        x[11] = torch.linspace(-3.3e38, 3.3e38, 64)
    x = x.to(dtype)
    cache = sq.QuantizedCache.empty(3, 1, 4, 64, formats(sq, bits))
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda()
    args = (table, torch.tensor([12], dtype=torch.int32).cuda(), starts_of([12]).cuda())
    sq.squant_cache_write(x.cuda(), (-x).cuda(), cache, *args)
    k, v = sq.squant_cache_read(cache, *args, 12, F32)
    for got, src in ((k, x), (v, -x)):
        c, s = quantise(src, bits)
        want = values(c, s).float()
        assert torch.equal(got.cpu().isnan(), want.isnan())
        assert torch.equal(got.cpu().nan_to_num(), want.nan_to_num())


def attend(sq, seed, lengths, new, heads, kv, dim, page, dtype, bits, wider=0, one_each=False, pad=0, scale=None):
    gen = torch.Generator().manual_seed(seed)
    pages, table = layout(gen, lengths, page, wider=wider)
    cache, host = filled(sq, gen, pages, kv, page, dim, bits)
    rows = sum(new) + pad
    q = (torch.randn(rows, heads, dim, generator=gen) * torch.rand(rows, 1, 1, generator=gen) * 2).to(dtype)
    lens = torch.tensor(lengths, dtype=torch.int32)
    starts = None if one_each else starts_of(new).cuda()
    out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), lens.cuda(), starts, scale)
    check(out, q, host, table, lengths, new, page, dtype, bits, dim ** -0.5 if scale is None else scale)
    return q, cache, host, table, lens, out


def check(out, q, host, table, lengths, new, page, dtype, bits, scale):
    """8 bits of 16-bit calls: elements of keys and values are rounded to 11 bits; weights always (binary32: 22, which is within the
    2^-20 that a weight may be off)."""
    r = 0
    rounded = 2.0 ** -11 if bits == 8 and dtype != F32 else 0.0 if dtype != F32 else 2.0 ** -22
    weight = F16 if dtype != F32 else F32
    for b, (n, m) in enumerate(zip(new, lengths)):
        p, s = slots_of(table, page, b, 0, m)
        k, v = (values(host[2 * i][p, :, s], host[2 * i + 1][p, :, s]) for i in range(2))
        ref = attention64(q[r:r + n].double(), k, v, scale, True, weight, key_error=rounded, value_error=rounded, floor=FLOOR)
        if dtype == BF16:  # weights of 11 bits, an output of 8
            ref["out_tol"] += 2.0 ** -8 * ref["out"].abs()
        close(out[r:r + n], ref, "out", f"sequence {b} of {lengths}, {new} new, page {page}")
        r += n
    assert (out[r:] == 0).all()


SHAPES = [(32, 8, 128, 16), (4, 4, 64, 24), (28, 4, 128, 64), (3, 1, 96, 17), (16, 2, 256, 32), (20, 1, 192, 48), (8, 8, 32, 7), (2, 2, 64, 1)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv,dim,page", SHAPES)
def test_attention_of_one_token(sq, heads, kv, dim, page, dtype, bits):
    lengths = [1, 33, 257, 64, 31]
    attend(sq, dim, lengths, [1] * 5, heads, kv, dim, page, dtype, bits, one_each=True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv,dim,page", SHAPES)
def test_attention_of_a_few_tokens(sq, heads, kv, dim, page, dtype, bits):
    lengths, new = [5, 40, 0, 131, 64, 3], [5, 3, 0, 8, 1, 7]  # the last has more rows than tokens: four see nothing
    q, cache, host, table, lens, out = attend(sq, dim + 1, lengths[:5], new[:5], heads, kv, dim, page, dtype, bits, pad=3)
    gen = torch.Generator().manual_seed(5)
    pages, table = layout(gen, [3], page)
    cache, host = filled(sq, gen, pages, kv, page, dim, bits)
    q = torch.randn(7, heads, dim, generator=gen).to(dtype)
    out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), torch.tensor([3], dtype=torch.int32).cuda(), starts_of([7]).cuda())
    check(out, q, host, table, [3], [7], page, dtype, bits, dim ** -0.5)
    assert (out[:4] == 0).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 50, 128])
def test_long_sequences_are_split(sq, page, dtype, bits):
    attend(sq, page, [3000, 1, 1025, 255], [1, 1, 1, 1], 8, 2, 128, page, dtype, bits, one_each=True)
    attend(sq, page, [2100, 300, 513], [2, 0, 5], 8, 2, 64, page, dtype, bits, wider=40, pad=2)


def test_many_rows(sq):
    """A chunk of a prompt: more rows than one pass takes."""
    attend(sq, 21, [300, 77], [90, 77], 8, 2, 64, 16, BF16, 4)
    attend(sq, 22, [70], [40], 4, 4, 256, 32, F16, 8)


def test_scales_of_any_size(sq):
    """Scales far beyond binary16's range, and within a block a factor of 2^20 apart."""
    for power in (-60, 60):
        gen = torch.Generator().manual_seed(23)
        pages, table = layout(gen, [300], 16)
        cache, host = filled(sq, gen, pages, 2, 16, 64, 4)
        host[1] *= 2.0 ** -power  # keys the other way: scores stay
        host[3] *= 2.0 ** power
        host[3][::3] *= 2.0 ** -20
        cache = sq.QuantizedCache(*(t.cuda() for t in host))
        q = (torch.randn(1, 4, 64, generator=gen) * 2.0 ** power).float()
        for dtype in (F32, BF16):
            qt = q.to(dtype)
            out = sq.squant_cache_attention(qt.cuda(), cache, table.cuda(), torch.tensor([300], dtype=torch.int32).cuda())
            check(out, qt, host, table, [300], [1], 16, dtype, 4, 0.125)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_hidden_slots(sq, dtype, bits):
    """NaN scales behind the sequence's end, in other pages, and at later new tokens reach no row that does not see them."""
    lengths, new, page = [45, 300], [4, 2], 16
    q, cache, host, table, lens, out = attend(sq, 31, lengths, new, 8, 2, 64, page, dtype, bits)
    cache = sq.QuantizedCache(*(t.clone() for t in cache))
    used = torch.zeros(cache.key_scales.shape[0], page, dtype=torch.bool)
    for b, m in enumerate(lengths):
        p, s = slots_of(table, page, b, 0, m)
        used[p, s] = True
    for t in (cache.key_scales, cache.value_scales):
        t[(~used)[:, None, :].expand(-1, 2, -1).cuda()] = math.nan
    again = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), lens.cuda(), starts_of(new).cuda())
    assert torch.equal(again, out)
    for value in (math.nan, math.inf):
        p, s = slots_of(table, page, 0, 43, 45)  # the last two tokens of the first sequence
        cache.key_scales[p.cuda(), :, s.cuda()] = value
        cache.value_scales[p.cuda(), :, s.cuda()] = value
        again = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), lens.cuda(), starts_of(new).cuda())
        check(again[:2], q[:2], host, table, [43], [2], page, dtype, bits, 0.125)
        assert again[2:4].isnan().any(-1).all()
        check(again[4:], q[4:], host, table[1:], lengths[1:], new[1:], page, dtype, bits, 0.125)


def test_missing_pages(sq):
    """A table's entry that is no page, and a length beyond the table: NaN for that sequence, nothing written, others as they are."""
    page = 16
    q, cache, host, table, lens, out = attend(sq, 32, [40, 40, 40, 500], [1, 1, 1, 1], 4, 2, 64, page, BF16, 4, one_each=True)
    broken = table.clone()
    broken[0, 1], broken[1, 0] = -1, cache.key_codes.shape[0]
    lens2 = lens.clone()
    lens2[2] = table.shape[1] * page + 1
    args = (broken.cuda(), lens2.cuda())
    again = sq.squant_cache_attention(q.cuda(), cache, *args)
    assert again[:3].isnan().all() and torch.equal(again[3], out[3])
    k = torch.randn(4, 2, 64, device="cuda", dtype=BF16)
    before = [t.clone() for t in cache]
    far = torch.tensor([20, 10, table.shape[1] * page + 1, 0], dtype=torch.int32).cuda()
    sq.squant_cache_write(k, k, cache, broken.cuda(), far)
    assert all(torch.equal(a.view(torch.int8), b.view(torch.int8)) for a, b in zip(cache, before))
    read, _ = sq.squant_cache_read(cache, broken.cuda(), far, None, 4, F16)
    assert read[:3].isnan().all() and (read[3] == 0).all()


def test_far_offsets(sq):
    """Pages whose bytes lie beyond 2^32 of the cache's beginning."""
    heads, page, dim = 8, 128, 128
    pages = 2 ** 32 // (heads * page * dim) + 40
    cache = sq.QuantizedCache.empty(pages, heads, page, dim, sq.OUT_INT8)
    gen = torch.Generator().manual_seed(33)
    lengths = [200, 129]
    table = torch.tensor([[pages - 1, pages - 3], [pages - 20, 0]], dtype=torch.int32)
    k, v = (torch.randn(sum(lengths), heads, dim, generator=gen).to(BF16) for _ in range(2))
    args = (table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda())
    sq.squant_cache_write(k.cuda(), v.cuda(), cache, *args, starts_of(lengths).cuda())
    got = sq.squant_cache_read(cache, *args, starts_of(lengths).cuda(), sum(lengths), BF16)
    for a, b in zip(got, (k, v)):
        assert torch.equal(a.cpu(), values(*quantise(b, 8)).to(BF16))
    q = torch.randn(2, 16, dim, generator=gen).to(BF16)
    out = sq.squant_cache_attention(q.cuda(), cache, *args)
    r = 0
    for b, m in enumerate(lengths):
        ref = attention64(q[b:b + 1].double(), values(*quantise(k[r:r + m], 8)), values(*quantise(v[r:r + m], 8)), dim ** -0.5, True, BF16,
                          key_error=2.0 ** -11, value_error=2.0 ** -11, floor=FLOOR)
        close(out[b:b + 1], ref, "out")
        r += m


def test_a_server(sq):
    """Prompts attend among themselves, go into the cache, and tokens follow one by one: written, then attending, as a captured
    graph that is replayed while the sequences grow; against attention over the values that the cache holds."""
    heads, kv, dim, page, bits = 8, 2, 64, 16, 4
    gen = torch.Generator().manual_seed(34)
    prompts, steps = [50, 3, 31], 20
    pages, table = layout(gen, [n + steps for n in prompts], page)
    cache = sq.QuantizedCache.empty(pages, kv, page, dim)
    x = torch.randn(sum(prompts), (heads + 2 * kv), dim, generator=gen).to(BF16).cuda()
    starts, lens = starts_of(prompts).cuda(), torch.tensor(prompts, dtype=torch.int32).cuda()
    tab = table.cuda()
    sq.squant_attention(x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:], starts)
    sq.squant_cache_write(x[:, heads:heads + kv], x[:, heads + kv:], cache, tab, lens, starts)
    held = [[t[a:b].cpu() for a, b in zip(starts.tolist(), starts.tolist()[1:])] for t in (x[:, heads:heads + kv], x[:, heads + kv:])]
    new = torch.zeros(3, heads + 2 * kv, dim, dtype=BF16, device="cuda")

    def step():
        sq.squant_cache_write(new[:, heads:heads + kv], new[:, heads + kv:], cache, tab, lens)
        return sq.squant_cache_attention(new[:, :heads], cache, tab, lens)
    lens.add_(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(steps):
        new.copy_(torch.randn(new.shape, generator=gen).to(BF16))
        torch.cuda.synchronize()
        graph.replay()
        for j, at in ((0, heads), (1, heads + kv)):
            for b in range(3):
                held[j][b] = torch.cat((held[j][b], new[b:b + 1, at:at + kv].cpu()))
        if i % 5 == 0 or i == steps - 1:
            eager = sq.squant_cache_attention(new[:, :heads], cache, tab, lens)
            assert torch.equal(eager, out)
            for b in range(3):
                k, v = (values(*quantise(held[j][b], bits)) for j in range(2))
                ref = attention64(new[b:b + 1, :heads].double().cpu(), k, v, dim ** -0.5, True, BF16, floor=FLOOR)
                close(out[b:b + 1], ref, "out", f"step {i}")
        lens.add_(1)


def test_graphs_with_workspaces_of_their_own(sq):
    """Two captured graphs of split calls, replayed in turn and with eager calls between."""
    sides = []
    for seed in (41, 42):
        q, cache, host, table, lens, out = attend(sq, seed, [1500, 700], [1, 1], 8, 2, 64, 16, BF16, 4, one_each=True)
        qg, tg, lg = q.cuda(), table.cuda(), lens.cuda()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            held = sq.squant_cache_attention(qg, cache, tg, lg)
        sides.append((graph, held, out, (qg, cache, tg, lg)))
    for _ in range(3):
        for graph, held, out, args in sides:
            held.zero_()
            graph.replay()
        for graph, held, out, args in sides:
            assert torch.equal(held, out) and torch.equal(sq.squant_cache_attention(*args), out)


def test_streams_outputs_and_strides(sq):
    q, cache, host, table, lens, out = attend(sq, 43, [700, 30], [1, 1], 8, 2, 64, 16, BF16, 4, one_each=True)
    buf = torch.full((2, 8 * 64 + 9), math.nan, dtype=BF16, device="cuda")
    view = buf[:, 3:3 + 512].unflatten(1, (8, 64))
    qs = torch.full((2, 8 * 64 + 7), math.nan, dtype=BF16, device="cuda")
    qv = qs[:, 1:513].unflatten(1, (8, 64))
    qv.copy_(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sq.squant_cache_attention(qv, cache, table.cuda(), lens.cuda(), out=view, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert got.data_ptr() == view.data_ptr() and torch.equal(view, out)
    assert buf[:, :3].isnan().all() and buf[:, 515:].isnan().all()


def test_empty(sq):
    cache = sq.QuantizedCache.empty(2, 2, 16, 64)
    ints = dict(dtype=torch.int32, device="cuda")
    table, lens = torch.zeros(0, 3, **ints), torch.zeros(0, **ints)
    q = torch.zeros(0, 4, 64, dtype=BF16, device="cuda")
    assert sq.squant_cache_attention(q, cache, table, lens).shape == (0, 4, 64)
    sq.squant_cache_write(q[:, :2], q[:, :2], cache, table, lens)
    q = torch.ones(3, 4, 64, dtype=BF16, device="cuda")
    starts = torch.zeros(1, **ints)
    assert (sq.squant_cache_attention(q, cache, table, lens, starts) == 0).all()  # padding only
    none = torch.zeros(3, 0, **ints)
    assert (sq.squant_cache_attention(q, cache, none, torch.zeros(3, **ints)) == 0).all()


def test_refusals(sq):
    cache = sq.QuantizedCache.empty(4, 2, 16, 64)
    ints = dict(dtype=torch.int32, device="cuda")
    table, lens, starts = torch.zeros(2, 2, **ints), torch.ones(2, **ints), torch.tensor([0, 1, 2], **ints)
    q = torch.zeros(2, 4, 64, dtype=BF16, device="cuda")
    k = torch.zeros(2, 2, 64, dtype=BF16, device="cuda")
    eight = sq.QuantizedCache.empty(4, 2, 16, 64, sq.OUT_INT8)
    mixed = sq.QuantizedCache(cache.key_codes, cache.key_scales, eight.value_codes, eight.value_scales)
    bad = [lambda: sq.squant_cache_attention(q[:, :3], cache, table, lens), lambda: sq.squant_cache_attention(q[:, :, :32], cache, table, lens),
           lambda: sq.squant_cache_attention(q, mixed, table, lens), lambda: sq.squant_cache_attention(q, cache, table.long(), lens),
           lambda: sq.squant_cache_attention(q, cache, table, lens[:1]), lambda: sq.squant_cache_attention(q, cache, table, lens, starts[:2]),
           lambda: sq.squant_cache_attention(q[:1], cache, table, lens), lambda: sq.squant_cache_attention(q, cache, table.cpu(), lens),
           lambda: sq.squant_cache_attention(q.double(), cache, table, lens), lambda: sq.squant_cache_attention(q.cpu(), cache, table, lens),
           lambda: sq.squant_cache_attention(q, cache, table[:, ::2], lens), lambda: sq.squant_cache_attention(q, cache, table, lens, out=q[:, :2]),
           lambda: sq.squant_cache_attention(q, cache._replace(key_scales=cache.key_scales.float()), table, lens),
           lambda: sq.squant_cache_attention(q, cache._replace(key_codes=cache.key_codes[:, :, ::2]), table, lens),
           lambda: sq.squant_cache_write(k, k[:1], cache, table, lens), lambda: sq.squant_cache_write(k, k.half(), cache, table, lens),
           lambda: sq.squant_cache_write(q, q, cache, table, lens), lambda: sq.squant_cache_write(k[..., :32], k[..., :32], cache, table, lens),
           lambda: sq.squant_cache_read(cache, table, lens, starts, 2, torch.float64), lambda: sq.squant_cache_read(cache, table, lens, None, 3, BF16),
           lambda: sq.squant_cache_read(cache, table, lens, None, 2, BF16, k=k[:1]), lambda: sq.QuantizedCache.empty(2, 1, 16, 48),
           lambda: sq.QuantizedCache.empty(2, 1, 16, 64, sq.OUT_F32)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(sq.SQuantError):
        sq.squant_cache_attention(q, cache, table, lens, scale=-1.0)


@pytest.mark.parametrize("one_each", [True, False])
def test_many_sequences(sq, one_each):
    for sequences in (63, 64, 65, 300):
        lengths = [(11 * i) % 40 + 1 for i in range(sequences)]
        new = [1 if one_each else min((3 * i) % 4, lengths[i]) for i in range(sequences)]
        attend(sq, sequences, lengths, new, 4, 2, 32, 16, BF16, 4, one_each=one_each, pad=0 if one_each else 2)


@pytest.mark.parametrize("sequences", [255, 256, 700])
def test_rows_of_many_sequences(sq, sequences):
    gen = torch.Generator().manual_seed(sequences)
    lengths = [(5 * i) % 17 for i in range(sequences)]
    new = [min((3 * i) % 5, lengths[i]) for i in range(sequences)]
    pages, table = layout(gen, lengths, 8)
    cache = sq.QuantizedCache.empty(pages, 2, 8, 64, sq.OUT_INT8)
    k, v = (torch.randn(sum(new) + 4, 2, 64, generator=gen).to(F16) for _ in range(2))
    args = (table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts_of(new).cuda())
    sq.squant_cache_write(k.cuda(), v.cuda(), cache, *args)
    for got, x in zip(sq.squant_cache_read(cache, *args, sum(new) + 4, F32), (k, v)):
        want = values(*quantise(x, 8)).float()
        want[sum(new):] = 0
        assert torch.equal(got.cpu(), want)
    r = 0
    for b, (n, m) in enumerate(zip(new, lengths)):  # and in the slots that they belong to
        p, s = slots_of(table, 8, b, m - n, m)
        codes, scales = quantise(v[r:r + n], 8)
        assert torch.equal(cache.value_codes.cpu()[p, :, s], codes)
        r += n


def test_broken_starts(sq):
    """Starts that fall, are negative or beyond the rows: what is computed is anything, in the buffers given."""
    q, cache, host, table, lens, out = attend(sq, 61, [600, 90, 40], [9, 2, 1], 4, 2, 64, 16, BF16, 4)
    rows = q.shape[0]
    for broken in ([0, 9, 3, 12], [4, -7, 90, 2], [0, 10 ** 9, 20, 2 ** 31 - 1], [12, 8, 4, 0]):
        starts = torch.tensor(broken, dtype=torch.int32).cuda()
        bufs = [torch.full((rows + 2, h, 64), 7.0, dtype=BF16, device="cuda") for h in (4, 2, 2)]
        sq.squant_cache_attention(q.cuda(), cache, table.cuda(), lens.cuda(), starts, out=bufs[0][1:-1])
        sq.squant_cache_read(cache, table.cuda(), lens.cuda(), starts, rows, BF16, k=bufs[1][1:-1], v=bufs[2][1:-1])
        assert all((b[0] == 7).all() and (b[-1] == 7).all() for b in bufs)


def test_overlaps(sq):
    q, cache, host, table, lens, out = attend(sq, 62, [40, 700], [1, 1], 4, 2, 64, 16, BF16, 8, one_each=True)
    qg, args = q.cuda(), (table.cuda(), lens.cuda())
    got = sq.squant_cache_attention(qg, cache, *args, out=qg)
    assert got is qg and torch.equal(qg, out)
    pair = torch.empty(2, 4, 64, dtype=BF16, device="cuda")
    k, v = sq.squant_cache_read(cache, *args, None, 2, BF16, k=pair[:, :2], v=pair[:, 2:])
    for a, b in zip((k, v), sq.squant_cache_read(cache, *args, None, 2, BF16)):
        assert torch.equal(a, b)
    inside = cache.key_codes.view(torch.uint8).flatten()[:2 * 4 * 64 * 2].view(BF16).view(2, 4, 64)
    wide = torch.zeros(3, 4, 64, dtype=BF16, device="cuda")
    before = [t.clone() for t in cache]
    bad = [lambda: sq.squant_cache_attention(wide[:2], cache, *args, out=wide[1:]), lambda: sq.squant_cache_attention(qg, cache, *args, out=inside),
           lambda: sq.squant_cache_read(cache, *args, None, 2, BF16, k=pair[:, :2], v=pair[:, 1:3]),
           lambda: sq.squant_cache_read(cache, *args, None, 2, BF16, v=inside[:, :2])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    assert all(torch.equal(a.view(torch.int8), b.view(torch.int8)) for a, b in zip(cache, before))


def test_two_streams_at_once(sq):
    sides = [torch.cuda.Stream() for _ in range(2)]
    work = []
    for i in range(2):
        q, cache, host, table, lens, out = attend(sq, 63 + i, [3000, 1700], [1, 1], 8, 2, 64, 16, BF16, 4, one_each=True)
        work.append((q.cuda(), cache, table.cuda(), lens.cuda(), out))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i, (q, cache, table, lens, out) in enumerate(work):
            got[i].append(sq.squant_cache_attention(q, cache, table, lens, stream=sides[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, work[i][4]) for g in got[i])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("scale", [0.0, 1e-45, 1e-38, 1e-3, 1.0])
def test_scales_of_scores(sq, scale, dtype, bits):
    """0, subnormal and ordinary ones; lengths that end inside a block, and a sequence that is split."""
    attend(sq, 71, [1, 33, 70, 1100], [1, 1, 1, 1], 8, 2, 64, 16, dtype, bits, one_each=True, scale=scale)
    attend(sq, 72, [45, 3, 130], [4, 3, 0], 4, 4, 96, 24, dtype, bits, pad=2, scale=scale)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("power", [-7, -14, -100])
def test_zero_keys_and_small_queries(sq, power, dtype, bits):
    """Keys of zero scales, all of a sequence's or its first ones, and queries whose products with them leave binary32: the mean of
    the values, or the later keys' softmax."""
    gen = torch.Generator().manual_seed(73)
    lengths, page = [1, 40, 75, 700], 16
    pages, table = layout(gen, lengths, page)
    cache, host = filled(sq, gen, pages, 2, page, 128, bits)
    for b, zeros in enumerate((1, 40, 64, 640)):
        p, s = slots_of(table, page, b, 0, zeros)
        host[1][p, :, s] = 0.0
    cache = sq.QuantizedCache(*(t.cuda() for t in host))
    q = (torch.randn(4, 8, 128, generator=gen) * 2.0 ** power).to(dtype)
    out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda())
    check(out, q, host, table, lengths, [1] * 4, page, dtype, bits, 128 ** -0.5)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_largest_scale_of_scores(sq, dtype):
    """A scale whose product with log2(e) leaves binary32: scores of 0 stay 0, over a cache and over prompts."""
    scale = torch.finfo(F32).max
    gen = torch.Generator().manual_seed(74)
    pages, table = layout(gen, [37], 16)
    cache, host = filled(sq, gen, pages, 2, 16, 64, 4)
    q = torch.zeros(1, 4, 64, dtype=dtype)
    out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), torch.tensor([37], dtype=torch.int32).cuda(), scale=scale)
    check(out, q, host, table, [37], [1], 16, dtype, 4, scale)
    v = torch.randn(37, 2, 64, generator=gen).to(dtype)
    out, lse = sq.squant_attention(q.cuda(), v.cuda(), v.cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda(),
                                   torch.tensor([0, 37], dtype=torch.int32).cuda(), scale=scale)
    ref = attention64(q.double(), v.double(), v.double(), scale, True, dtype)
    close(out, ref, "out")
    close(lse, ref, "lse")
    for got in sq.squant_attention_backward(torch.zeros_like(out), q.cuda(), v.cuda(), v.cuda(), out, lse, torch.tensor([0, 1], dtype=torch.int32).cuda(),
                                            torch.tensor([0, 37], dtype=torch.int32).cuda(), scale=scale):
        assert (got == 0).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("which", ["key", "value"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_one_broken_scale(sq, value, which, dtype, bits):
    """A token with one scale of its keys, or of its values, that is no number: rows that see it are NaN throughout, also where all products
    with an infinite key are minus infinity; others are as they are."""
    lengths, new, page = [45, 300], [4, 2], 16
    gen = torch.Generator().manual_seed(75)
    pages, table = layout(gen, lengths, page)
    cache, host = filled(sq, gen, pages, 2, page, 64, bits)
    p, s = slots_of(table, page, 0, 43, 44)
    if bits == 4:
        host[0][p, :, s] = 0xdd  # -3, -3
    else:
        host[0][p, :, s] = -3
    cache = sq.QuantizedCache(*(t.cuda() for t in host))
    q = (torch.randn(6, 8, 64, generator=gen).abs() + 0.5).to(dtype)
    args = (table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts_of(new).cuda())
    out = sq.squant_cache_attention(q.cuda(), cache, *args)
    check(out, q, host, table, lengths, new, page, dtype, bits, 0.125)
    scales = cache.key_scales if which == "key" else cache.value_scales
    for heads, group in ((slice(0, 1), 1), (slice(0, 2), 0)):
        scales[p.cuda(), heads, s.cuda(), group] = value
        again = sq.squant_cache_attention(q.cuda(), cache, *args)
        seen = slice(0, 4 * heads.stop)  # query heads of those key heads
        assert again[2:4, seen].isnan().all()
        assert torch.equal(again[2:4, 4 * heads.stop:], out[2:4, 4 * heads.stop:])
        close_rows = again.clone()
        close_rows[2:4] = out[2:4]
        check(close_rows, q, host, table, lengths, new, page, dtype, bits, 0.125)


@pytest.mark.parametrize("page,width", [(16, 3), (7, 5), (16, 0), (16, 200)])
def test_rows_that_see_beyond_the_table(sq, page, width):
    """Rows of a sequence that is longer than its table are NaN where they see a token beyond it, and only there; rows that see nothing are 0."""
    gen = torch.Generator().manual_seed(76)
    capacity = page * width
    pages, table = layout(gen, [max(capacity, 1)], page)
    table = table[:, :width].contiguous()
    cache, host = filled(sq, gen, pages, 2, page, 64, 4)
    for new, beyond in ((1, 1), (5, 2), (5, 5), (5, 9), (40, 3)):
        length = capacity + beyond
        q = torch.randn(new, 4, 64, generator=gen).to(BF16)
        out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), torch.tensor([length], dtype=torch.int32).cuda(), starts_of([new]).cuda())
        whole = max(new - beyond, 0)  # rows that end within the table
        assert out[whole:].isnan().all()
        nothing = min(max(new - length, 0), whole)
        assert (out[:nothing] == 0).all()
        if whole > nothing:
            check(out[nothing:whole], q[nothing:whole], host, table, [capacity], [whole - nothing], page, BF16, 4, 0.125)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,power", [(BF16, 24), (BF16, 60), (F16, 24), (F32, 24), (F32, 60)])
def test_scores_of_any_size(sq, dtype, power, bits, sign):
    """Scores so far apart that a row's output is the value of its largest one, where a product's rounding is more than a weight's exponent."""
    gen = torch.Generator().manual_seed(78)
    lengths, new, page, half = [70, 1100], [3, 1], 16, power // 2
    pages, table = layout(gen, lengths, page)
    cache, host = filled(sq, gen, pages, 1, page, 64, bits)
    host[0].zero_()
    host[0][..., 0] = 1
    counts = []
    for b, m in enumerate(lengths):
        p, s = slots_of(table, page, b, 0, m)
        counts.append(torch.randperm(m, generator=gen) % 97 + 1)
        host[1][p, :, s, 0] = (sign * counts[-1].float() * 2.0 ** (half - 3)).to(BF16)[:, None]
        for t in host[2:]:
            t[p, :, s] = torch.stack([t[p[counts[-1] == c][0], :, s[counts[-1] == c][0]] for c in counts[-1]])  # equal ones have equal values
    cache = sq.QuantizedCache(*(t.cuda() for t in host))
    q = torch.zeros(4, 2, 64, dtype=dtype)
    q[..., 0] = 2.0 ** (power - half + 2)
    out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts_of(new).cuda())
    for r, (b, sees) in enumerate(((0, 68), (0, 69), (0, 70), (1, 1100))):
        p, s = slots_of(table, page, b, 0, sees)
        best = (sign * counts[b][:sees]).argmax()
        v = values(host[2][p, :, s], host[3][p, :, s])[best]
        # elements of 11 bits (a remainder in the other types); weights and their sum; the output
        tol = (2.0 ** -20 + 2.0 ** -11 * 2 + torch.finfo(dtype).eps / 2) * v.abs()
        assert ((out[r].cpu().double() - v).abs() <= tol).all(), r


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("power", [108, 118, 121])
def test_large_values(sq, power, dtype, bits):
    """Values whose products with the weights' unit leave binary32, and their means do not."""
    gen = torch.Generator().manual_seed(79)
    lengths, new, page = [7, 600], [2, 1], 16
    pages, table = layout(gen, lengths, page)
    cache, host = filled(sq, gen, pages, 2, page, 64, bits)
    host[1].mul_(2.0 ** -12)  # scores next to each other
    host[3].fill_(2.0 ** (power - (0 if bits == 4 else 4)))  # 8 bits: codes to 127
    if power > 118:  # the sum of a sequence's values would leave binary32 too
        lengths = [7, 12]
        table = table[:, :1].contiguous()
    cache = sq.QuantizedCache(*(t.cuda() for t in host))
    q = torch.randn(3, 4, 64, generator=gen).to(dtype)
    out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts_of(new).cuda())
    check(out, q, host, table, lengths, new, page, dtype, bits, 0.125)
    assert out.isfinite().all()


def later_tokens(sq, lengths, new, page, dim, heads, kv, wider, power, which, dtype, bits):
    """New tokens whose scales are each 2^power times those of the one before: a row is as good as it is without the tokens behind it.

    Bound beside check's: an element is off by at most 2^-24 of the largest that the row sees, and a score by that for its key."""
    gen = torch.Generator().manual_seed(77)
    pages, table = layout(gen, lengths, page, wider=wider)
    cache, host = filled(sq, gen, pages, kv, page, dim, bits)
    for b, (m, n) in enumerate(zip(lengths, new)):
        for i in range(1, n):
            p, s = slots_of(table, page, b, m - n + i, m - n + i + 1)
            for j, name in ((1, "keys"), (3, "values")):
                if which in (name, "both"):
                    host[j][p, :, s] = 2.0 ** (power * i - 4)
    cache = sq.QuantizedCache(*(t.cuda() for t in host))
    q = (torch.randn(sum(new), heads, dim, generator=gen) * 0.25).to(dtype)
    out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts_of(new).cuda())
    scale, group = dim ** -0.5, heads // kv
    rounded = 2.0 ** -11 if bits == 8 and dtype != F32 else 0.0 if dtype != F32 else 2.0 ** -22
    r = 0
    for b, (m, n) in enumerate(zip(lengths, new)):
        for i in range(n):
            sees = m - n + i + 1
            p, s = slots_of(table, page, b, 0, sees)
            if any(not host[x][p, :, s].isfinite().all() for x in (1, 3)):
                assert out[r].isnan().all()
                r += 1
                continue
            k, v = (values(host[2 * x][p, :, s], host[2 * x + 1][p, :, s]) for x in range(2))
            row = q[r:r + 1].double()
            ref = attention64(row, k, v, scale, True, F16 if dtype != F32 else F32, key_error=rounded, value_error=rounded, floor=FLOOR)
            worst = scale * 2.0 ** -24 * k.abs().amax((0, 2)).repeat_interleave(group) * row.abs().sum(-1)[0]  # of a score
            most = v.abs().amax((0, 2)).repeat_interleave(group)
            ref["out_tol"] += ((2.0 ** -24 + 4 * worst) * most)[None, :, None]
            if dtype == BF16:
                ref["out_tol"] += 2.0 ** -8 * ref["out"].abs()
            held = max(k.abs().max(), v.abs().max()) < 2.0 ** 128  # 127 * 2^121 is beyond binary32, and no token written holds it
            if held and (dtype != F16 or most.max() < 6e4):  # binary16's range
                close(out[r:r + 1], ref, "out", f"row {i} of {n}, {sees} tokens")
            r += 1


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("which", ["keys", "values", "both"])
@pytest.mark.parametrize("power", [3, 12, 30, 60, -12, -30])  # 60 times four is beyond bfloat16: the scale is infinite, the rows that see it NaN
def test_later_tokens_of_other_sizes(sq, power, which, dtype, bits):
    later_tokens(sq, [45, 34, 3, 300], [4, 5, 3, 2], 16, 64, 8, 2, 0, power, which, dtype, bits)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("power", [4, 12, 25])
@pytest.mark.parametrize("lengths,new,page,dim,heads,kv,wider",
                         [([45, 700, 1030], [4, 5, 3], 16, 64, 8, 2, 90), ([45, 70], [4, 5], 7, 96, 3, 3, 0), ([514, 1200], [5, 6], 24, 32, 4, 1, 40),
                          ([70, 40], [6, 6], 32, 128, 8, 2, 0), ([520, 33], [6, 6], 64, 128, 8, 1, 40), ([90], [9], 16, 256, 4, 2, 0),
                          ([80, 66], [9, 10], 50, 192, 2, 1, 0), ([100, 64], [28, 3], 16, 64, 4, 1, 60)])
def test_later_tokens_in_other_layouts(sq, lengths, new, page, dim, heads, kv, wider, power, dtype, bits):
    """Pieces of sequences, odd pages, two halves of 16 rows, sizes of head, more rows than a tile."""
    later_tokens(sq, lengths, new, page, dim, heads, kv, wider, power, "both", dtype, bits)


def test_many_sequences_of_a_wide_table(sq):
    """More pieces than the workspace's ceiling allows: stretches grow, and sequences lie in several of them all the same."""
    lengths = [(37 * i) % 200 + 1 for i in range(300)]
    lengths[7], lengths[251] = 9000, 4001
    attend(sq, 80, lengths, [1] * 300, 32, 2, 64, 16, BF16, 4, wider=9600, one_each=True)
    import ctypes
    A = sq.attention
    place = A.squant_paged_t(256, 256, None, 300, 563 + 9600)
    codes = A.squant_cache_t(256, 256, 256, 256, 10, 16, 2, 64, sq.OUT_INT4)
    assert A._lib().squant_cache_attention_workspace_bytes(300, 32, ctypes.byref(codes), ctypes.byref(place)) > 2 * 300 * 32 * 264


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("heads,dim", [(512, 256), (1365, 96), (4096, 32)])
def test_most_heads(sq, heads, dim, bits):
    gen = torch.Generator().manual_seed(heads)
    cache = sq.QuantizedCache.empty(3, heads, 2, dim, formats(sq, bits))
    args = (torch.tensor([[1, 2]], dtype=torch.int32).cuda(), torch.tensor([3], dtype=torch.int32).cuda(), starts_of([3]).cuda())
    k, v = (torch.randn(3, heads, dim, generator=gen).to(BF16) for _ in range(2))
    sq.squant_cache_write(k.cuda(), v.cuda(), cache, *args)
    for got, x in zip(sq.squant_cache_read(cache, *args, 3, F32), (k, v)):
        assert torch.equal(got.cpu(), values(*quantise(x, bits)).float())
    q = torch.randn(3, heads, dim, generator=gen).to(BF16)
    out = sq.squant_cache_attention(q.cuda(), cache, *args)
    some = torch.tensor([0, 1, heads // 2, heads - 1])
    rounded = 2.0 ** -11 if bits == 8 else 0.0
    ref = attention64(q[:, some].double(), values(*quantise(k[:, some], bits)), values(*quantise(v[:, some], bits)), dim ** -0.5, True, F16,
                      key_error=rounded, value_error=rounded, floor=FLOOR)
    ref["out_tol"] += 2.0 ** -8 * ref["out"].abs()
    close(out[:, some.cuda()], ref, "out")


def eleven_bits(x):
    """x (64 bits) rounded to 11 significant bits."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2.0 ** 11), e - 11)


def whole_elements(gen, dtype, which):
    """48 sequences of two tokens, 8 bits, whose output shows the last bits of their elements: (q, host cache, exact output [48, 1, 64], bound,
    output with elements of 11 bits)."""
    n, dim = 48, 64
    codes = [torch.zeros(n, 1, 2, dim, dtype=torch.int8) for _ in range(2)]
    scales = [(torch.randint(129, 255, (n, 1, 2, 2), generator=gen) * 2.0 ** -7).to(BF16) for _ in range(2)]
    q = torch.zeros(n, 1, dim, dtype=dtype)
    if which == "values":
        # equal weights, 2^14 each: the sum of the two values, which nearly cancel, is exact
        scales[1][:, :, 1] = scales[1][:, :, 0]
        first = torch.randint(100, 127, (n, 1, dim), generator=gen)
        codes[1][:, :, 0], codes[1][:, :, 1] = first.to(torch.int8), (torch.randint(-4, 5, (n, 1, dim), generator=gen) - first).to(torch.int8)
    else:
        # scores of about 2^9 next to each other, of different elements of the query; values 1 and -1
        codes[0][:, :, 0, 0], codes[0][:, :, 1, 40] = 127, 101
        k = values(codes[0], scales[0])
        a = 2.0 ** 12 / k[:, 0, 0, 0] * (1 + torch.rand(n, generator=gen).double() / 4)
        q[:, 0, 0] = a.to(dtype)
        q[:, 0, 40] = (q[:, 0, 0].double() * k[:, 0, 0, 0] / k[:, 0, 1, 40]).to(dtype)
        codes[1][:, :, 0], codes[1][:, :, 1], scales[1][:] = 1, -1, 1.0

    def run(of):
        k, v = of(values(codes[0], scales[0]))[:, 0], of(values(codes[1], scales[1]))[:, 0]
        s = 0.125 * (k @ q.double().transpose(1, 2))[..., 0]
        return (torch.softmax(s, 1)[..., None] * v).sum(1, keepdim=True)
    exact = run(lambda x: x)
    half = torch.finfo(dtype).eps / 2
    if which == "values":
        tol = half * exact.abs()  # one rounding
    else:
        # binary32 sums of products of 2^9 or less each, 24 steps; a weight is rounded (11 or 22 bits), the output once
        tol = torch.full_like(exact, 2 * 24 * 2.0 ** -23 * 2 * 640 + 2.0 ** -11 + 2.0 ** -20) + half * exact.abs()
    return q, [codes[0], scales[0], codes[1], scales[1]], exact, tol, run(eleven_bits)


@pytest.mark.parametrize("which", ["keys", "values"])
@pytest.mark.parametrize("dtype", [F16, F32])
def test_whole_elements_of_8_bits(sq, dtype, which):
    """Binary16 and binary32 calls multiply by all 15 bits of an element."""
    q, host, exact, tol, short = whole_elements(torch.Generator().manual_seed(82), dtype, which)
    assert ((short - exact).abs() > tol).double().mean() > 0.5  # elements of 11 bits would be seen
    cache = sq.QuantizedCache(*(t.cuda() for t in host))
    table, lens = torch.arange(48, dtype=torch.int32).view(48, 1).cuda(), torch.full((48,), 2, dtype=torch.int32).cuda()
    out = sq.squant_cache_attention(q.cuda(), cache, table, lens).cpu().double()
    assert ((out - exact).abs() <= tol).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_beyond_binary32(sq, dtype, bits):
    """A zero key among those whose scores are minus infinity in binary32: its value."""
    gen = torch.Generator().manual_seed(83)
    pages, table = layout(gen, [50], 16)
    cache, host = filled(sq, gen, pages, 1, 16, 64, bits)
    host[0].fill_(0x11 if bits == 4 else 1)
    host[1].fill_(-2.0 ** 100)
    p, s = slots_of(table, 16, 0, 20, 21)
    host[1][p, :, s] = 0.0
    cache = sq.QuantizedCache(*(t.cuda() for t in host))
    q = torch.full((1, 2, 64), 2.0 ** 100, dtype=dtype)
    out = sq.squant_cache_attention(q.cuda(), cache, table.cuda(), torch.tensor([50], dtype=torch.int32).cuda())
    want = values(host[2][p, :, s], host[3][p, :, s])[0]
    tol = (2.0 ** -11 + torch.finfo(dtype).eps / 2) * want.abs()
    assert ((out[0].cpu().double() - want).abs() <= tol).all()
