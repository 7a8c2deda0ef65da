"""Rows in 8 bits on the GPU, against their definition in 64 bits.

Tolerances count roundings (u = 2^-24 is half a step of fp32, relative; 2^-8 of bf16):
 - a scale max / 127: the quotient's and the store's, 2 u; with the norm the fp32 sum of squares as well: every square and every
   addition that a value passes through (at most 64 in a thread's own sum and 16 across the block) 1 u, halved by the root, and the
   root, the quotients and the gain's product: under 64 u.
 - a code is y / s rounded, y / s formed from at most four rounded operations on values up to 127: off by at most half a step
   and 127 * 4 u.
 - a product: the whole sum to fp32, two factors, bias and residual: 5 u of the sum of their magnitudes, and the result's type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF, F = torch.bfloat16, torch.float32


def rows_of(seed, rows, k, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, k), generator=g, device="cuda")
    return (x * torch.exp(2 * torch.randn((rows, 1), generator=g, device="cuda"))).to(dtype)


def check_codes(codes, scales, y, k, units):
    """codes and scales of the rows y (64 bits, finite)."""
    s = y.abs().amax(1) / 127
    assert codes.shape == (y.shape[0], -(-k // 128) * 128) and (codes[:, k:] == 0).all()
    assert ((scales.double() - s).abs() <= s * units * U + 2.0 ** -149).all()
    q = codes[:, :k].double()
    t = y / torch.where(s > 0, s, torch.ones_like(s))[:, None]
    assert q.abs().max() <= 127 and ((q - t).abs() <= 0.5 + 127 * 4 * U).all()


QUANTIZE = [(1, 1), (3, 1), (1, 7), (5, 64), (2, 127), (130, 128), (7, 129), (33, 500), (3, 511), (4, 512), (3, 513), (257, 1024), (9, 1025), (5, 2047),
            (300, 12544), (2, 8191), (2, 8193), (3, 16385), (1, 32769), (2, 65535), (1, 65536), (20000, 24), (9600, 1024)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,k", QUANTIZE)
def test_quantize(rows, k, dtype):
    import paper_2102_08481_amd as thia
    x = rows_of(rows + k, rows, k, dtype)
    check_codes(*thia.thia_quantize_rows(x), x.double(), k, 2)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,k", QUANTIZE)
def test_norm(rows, k, residual, dtype):
    import paper_2102_08481_amd as thia
    x, r = rows_of(rows + k, rows, k, dtype), rows_of(rows + k + 1, rows, k, dtype) if residual else None
    gain, eps = 0.5 + torch.rand(k, device="cuda"), 1e-3
    codes, scales, total = thia.thia_rms_norm_i8(x, gain, eps, r)
    h = x.double() + (r.double() if residual else 0)
    assert (total is None) == (not residual)
    if residual:
        assert torch.equal(total, (x.float() + r.float()).to(dtype))
        h = (x.float() + r.float()).double()   # the sum is held in fp32
    check_codes(codes, scales, h * gain.double() / torch.sqrt((h * h).mean(1, keepdim=True) + eps), k, 64)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("k", [5, 1000, 9000, 40000])
def test_rows_without_values_and_extreme_rows(k, dtype):
    """Rows of zeros, of the smallest and of the largest values, and rows with NaN or infinity among ordinary ones."""
    import paper_2102_08481_amd as thia
    x = rows_of(k, 12, k, dtype)
    x[1], x[3] = 0, 0
    x[3, k // 2] = 2.0 ** -133            # a single value, below the normal numbers
    x[4] = x[4].sign() * 3.0e38
    x[5] = x[5].sign() * 1.0e-38
    x[6] = x[6].sign() * 2.0e25           # squares beyond fp32
    x[7, k - 1], x[8, 0], x[9, k // 3] = float("nan"), float("inf"), -float("inf")
    x[10] = -0.0
    fine = torch.tensor([0, 1, 2, 3, 4, 5, 6, 10, 11], device="cuda")
    gain = 0.5 + torch.rand(k, device="cuda")
    for codes, scales, y, units in (
            thia.thia_quantize_rows(x) + (x.double(), 2),
            thia.thia_rms_norm_i8(x, gain, 1e-12)[:2] + (x.double() * gain.double() / torch.sqrt((x.double() ** 2).mean(1, keepdim=True) + 1e-12), 64)):
        check_codes(codes[fine], scales[fine], y[fine], k, units)
        assert scales[7:10].isnan().all() and (codes[7:10] == 0).all()
        assert scales[1] == 0 and scales[10] == 0


def test_norm_with_a_sum_that_overflows_or_cancels():
    import paper_2102_08481_amd as thia
    x = rows_of(1, 3, 777, F)
    r = rows_of(2, 3, 777, F)
    x[0, 3] = r[0, 3] = 3e38              # infinite as a sum
    r[1] = -x[1]                          # nothing left
    gain = torch.ones(777, device="cuda")
    codes, scales, total = thia.thia_rms_norm_i8(x, gain, 1e-6, r)
    assert torch.equal(total, x + r) and scales[0].isnan() and (codes[0] == 0).all() and scales[1] == 0 and (codes[1] == 0).all()
    h = (x + r)[2:].double()
    check_codes(codes[2:], scales[2:], h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6), 777, 64)


def test_norm_with_zero_and_large_gains():
    import paper_2102_08481_amd as thia
    x = rows_of(5, 4, 300, F)
    for gain in (torch.zeros(300, device="cuda"), torch.full((300,), -1e-30, device="cuda"), torch.full((300,), 1e30, device="cuda")):
        codes, scales, _ = thia.thia_rms_norm_i8(x * 1e-3, gain, 1e-6)
        h = (x * 1e-3).double()
        check_codes(codes, scales, h * gain.double() / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6), 300, 64)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("k", [5, 300, 2000, 9000, 40000])
def test_norm_with_gains_at_the_ends_of_fp32(k, dtype):
    """y is finite and its codes reach 127 whatever the gain's size: products of a value and a gain that leave fp32 on either side, also
    where the row's largest values have no gain.  The eps lies far below, near and far above the mean of the squares."""
    import paper_2102_08481_amd as thia
    x = rows_of(k + 3, 6, k, dtype)
    x[4] *= 2.0 ** -60
    x[5] *= 2.0 ** 60
    sign = torch.where(rows_of(1, 1, k, F)[0] > 0, 1.0, -1.0)
    for size in (1e-36, 1e-37, 1e-38, 2.0 ** -130, 2.0 ** -149, 1e38, 3.4e38):
        gain = sign * size
        for eps in (1e-38, 1.0, 1e38):
            codes, scales, _ = thia.thia_rms_norm_i8(x, gain, eps)
            h = x.double()
            check_codes(codes, scales, h * gain.double() / torch.sqrt((h * h).mean(1, keepdim=True) + eps), k, 64)
            assert (codes.abs().amax(1) == 127).all()
    some = torch.arange(k, device="cuda") % 4 == 0
    x[:, some] = x[:, some].sign() * 2.0 ** 126
    for size in (2.0 ** -100, 1.0, 3e38):   # (y's largest is 2^-186 or so times the gain: the codes hold where the scale no longer does)
        gain = torch.where(some, 0.0, size)
        codes, scales, _ = thia.thia_rms_norm_i8(x, gain, 1e-6)
        h = x.double()
        check_codes(codes, scales, h * gain.double() / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6), k, 64)
        assert (codes.abs().amax(1) == 127).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("k", [37, 3000, 20000])
def test_norm_of_unusual_rows_in_place(k, dtype):
    """Rows whose products or squares leave fp32, rows of zeros and rows that are no numbers between ordinary ones, the sum in place of
    either input or beside them."""
    import paper_2102_08481_amd as thia
    x, r = rows_of(k, 23, k, dtype), rows_of(k + 1, 23, k, dtype)
    for i, size in ((3, 2.0 ** -70), (4, 2.0 ** 70), (9, 0.0), (10, 2.0 ** -120), (16, 2.0 ** 120)):
        x[i] *= size
        r[i] *= size
    x[7, k // 2], r[12, 0] = float("inf"), float("nan")
    fine = torch.tensor([i for i in range(23) if i not in (7, 12)], device="cuda")
    for size in (1.0, 1e-37, 1e37):
        gain = (0.5 + torch.rand(k, device="cuda")) * size
        codes, scales, total = thia.thia_rms_norm_i8(x, gain, 1e-6, r)
        assert torch.equal(total[fine], (x.float() + r.float()).to(dtype)[fine]) and total[7, k // 2].isinf() and total[12, 0].isnan()
        h = (x.float() + r.float()).double()[fine]
        check_codes(codes[fine], scales[fine], h * gain.double() / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6), k, 64)
        assert scales[7].isnan() and scales[12].isnan() and (codes[7] == 0).all() and (codes[12] == 0).all()
        for target in (0, 1):
            y = [x.clone(), r.clone()]
            got = thia.thia_rms_norm_i8(y[0], gain, 1e-6, y[1], sum_out=y[target])
            assert torch.equal(got[0], codes) and torch.equal(got[1][fine], scales[fine]) and torch.equal(got[2][fine], total[fine])
            assert torch.equal(y[1 - target].isnan(), (x, r)[1 - target].isnan())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("k", [37, 1000, 4099])
def test_rows_with_pitches_on_odd_addresses_and_sums_in_place(k, dtype):
    import paper_2102_08481_amd as thia
    wide = rows_of(k, 19, 2 * k + 9, dtype)
    x, r = wide[:, 1:k + 1], wide[:, k + 3:2 * k + 3]
    gain = 0.5 + torch.rand(2 * k, device="cuda")[1:k + 1]
    want = thia.thia_rms_norm_i8(x.contiguous(), gain, 1e-6, r.contiguous())
    plain = thia.thia_quantize_rows(x.contiguous())
    assert all(torch.equal(a, b) for a, b in zip(thia.thia_quantize_rows(x), plain))
    room = torch.full((19, k + 5), 7, dtype=dtype, device="cuda")
    got = thia.thia_rms_norm_i8(x, gain, 1e-6, r, sum_out=room[:, 2:k + 2])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (room[:, :2] == 7).all() and (room[:, k + 2:] == 7).all()
    for target in (0, 1):   # the sum in place of either input
        again = wide.clone()
        x, r = again[:, 1:k + 1], again[:, k + 3:2 * k + 3]
        got = thia.thia_rms_norm_i8(x, gain, 1e-6, r, sum_out=(x, r)[target])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        kept = torch.ones_like(wide, dtype=torch.bool)
        kept[:, (1, k + 3)[target]:(k + 1, 2 * k + 3)[target]] = False
        assert torch.equal(again[kept], wide[kept])


def test_rows_behind_the_last_stay():
    import paper_2102_08481_amd as thia
    x = rows_of(3, 9, 200, BF)
    codes, scales = torch.full((12, 256), 5, dtype=torch.int8, device="cuda"), torch.full((12,), 5.0, device="cuda")
    thia.thia_quantize_rows(x, out=(codes[:9], scales[:9]))
    assert (codes[9:] == 5).all() and (scales[9:] == 5).all()
    want = thia.thia_quantize_rows(x)
    assert torch.equal(codes[:9], want[0]) and torch.equal(scales[:9], want[1])


def nearest_codes(x, k):
    """127 y / max to the nearest whole number, ties to even.  The quotient in 64 bits is exact at ties (254 y = (2 m + 1) max), and all
    others lie at least 2^-34 from one: with mantissas Y and M of up to 24 bits and quotients of 1/2 and more, |254 Y / 2^a - (2 m + 1) M| / 2 M
    with a whole Y 2^-a down to 2^-8."""
    y = x.double()
    most = y.abs().amax(1, keepdim=True)
    return torch.round(127 * y / torch.where(most > 0, most, torch.ones_like(most)))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("k", [8, 1000, 5000, 20000])
def test_codes_between_two_whole_numbers_go_to_the_even_one(k, dtype):
    """Half of a row's largest value lies between 63 and 64, whatever that value is: 64, for the codes of rows, the norm's with gain 1,
    and a layer's channels alike; and of bf16 rows every code is the nearest."""
    import paper_2102_08481_amd as thia
    m = torch.arange(128, 256, device="cuda").float()
    most = torch.cat([m * 2.0 ** e for e in (-118, -107, -60, -8, 0, 50, 93, 119)])
    x = (rows_of(k, len(most), k, F).clamp(-8, 8) / 8 * most[:, None]).to(dtype)
    x[:, 0], x[:, 3], x[:, 5] = most.to(dtype), (most / 2).to(dtype), (-most / 2).to(dtype)
    assert torch.equal(x[:, 3].double() * 2, most.double())
    q = thia.thia_quantize_rows(x)[0][:, :k].double()
    assert (q[:, 0] == 127).all() and (q[:, 3] == 64).all() and (q[:, 5] == -64).all()
    one = torch.ones(k, device="cuda")
    n = thia.thia_rms_norm_i8(x, one, 1e-6)[0][:, :k].double()
    assert torch.equal(n, q)
    want = nearest_codes(x, k)
    if dtype is BF:
        assert torch.equal(q, want)
    else:   # (the quotient is held in fp32: half a step of 2^-17 where it is largest)
        t = 127 * x.double() / most.double()[:, None]
        assert ((q - t).abs() <= 0.5 + 2.0 ** -18).all()
    # a layer's channels: seen through rows that have one code each
    codes = torch.eye(8, 128, device="cuda").to(torch.int8)
    fine = most < 2.0 ** 100   # (codes * scale of the others leave fp32)
    w = x[fine][:, :8].float().contiguous()
    layer = thia.thia_linear_i8_load(w)
    s = thia.thia_quantize_rows(w)[1]
    out = thia.thia_linear_i8_run(layer, codes, torch.ones(8, device="cuda"), out_f32=True)
    assert torch.equal(out, q[fine][:, :8].t().float().contiguous() * s)


# ---------------------------------------------------------------- the product
def layer_of(seed, n, k, low=-127):
    import paper_2102_08481_amd as thia
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    codes = torch.randint(low, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    scales, bias = 0.01 + torch.rand(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda") * 1000
    return thia.thia_linear_i8_load_codes(codes, scales, bias), codes, scales, bias


def codes_of(seed, rows, k, low=-127):
    """Codes with anything behind column k."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    codes = torch.randint(low, 128, (rows, -(-k // 128) * 128), generator=g, device="cuda", dtype=torch.int8)
    return codes, 0.01 + torch.rand(rows, generator=g, device="cuda")


def check_product(out, codes, scales, w, ws, bias, k, relu=False, residual=None):
    acc = torch.matmul(codes[:, :k].double(), w.double().t().contiguous())   # whole numbers below 2^53: exact
    part = acc * scales.double()[:, None] * ws.double()
    want, size = part + bias.double(), part.abs() + bias.double().abs()
    if residual is not None:
        want, size = want + residual.double(), size + residual.double().abs()
    if relu:
        want = want.clamp(min=0)
    off = (out.double() - want).abs()
    assert (off <= size * 5 * U * 1.001 + want.abs() * HALF[out.dtype] * 1.001).all(), float((off / size).max())


LINEAR = [(1, 1, 1), (1, 16, 64), (2, 130, 3), (1, 4096, 4096), (3, 4097, 100), (15, 1000, 33), (16, 1024, 1024), (17, 512, 96), (31, 65, 31), (32, 64, 32),
          (33, 128, 257), (63, 2000, 65), (64, 256, 64), (65, 300, 128), (100, 12544, 40), (127, 640, 129), (128, 128, 128), (300, 12544, 1024), (301, 384, 1000),
          (1000, 700, 8), (1021, 1024, 250), (2000, 1024, 100), (2048, 256, 2048), (4096, 1024, 512), (5000, 513, 511), (1, 65536, 8), (40, 65536, 40),
          (9600, 1024, 1024), (3000, 896, 2300), (20000, 64, 64), (70000, 16, 24), (2, 8, 300000)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,k,n", LINEAR)
def test_linear(rows, k, n, dtype):
    import paper_2102_08481_amd as thia
    layer, w, ws, b = layer_of(rows + n, n, k)
    codes, scales = codes_of(k, rows, k)
    out = thia.thia_linear_i8_run(layer, codes, scales, out_f32=dtype is F)
    assert out.dtype == dtype and tuple(out.shape) == (rows, n)
    check_product(out, codes, scales, w, ws, b, k)
    residual = rows_of(7, rows, n, dtype) * 1000
    check_product(thia.thia_linear_i8_run(layer, codes, scales, True, residual, dtype is F), codes, scales, w, ws, b, k, True, residual)


# ragged shapes that reach every tile: 16 x 16, 32 x 32, 32 x 64, 64 x 64, 96 x 64, 128 x 64, 128 x 128, 192 x 256, 256 x 256, the rings and
# phases with two, three and more K tiles
RAGGED = [(5, 200, 37), (700, 640, 130), (1003, 2000, 515), (2001, 1000, 1001), (1187, 12001, 1003), (2003, 12544, 1000), (2100, 100, 1999), (2001, 200, 1999),
          (3000, 257, 1030), (9001, 130, 1001), (2901, 300, 2001), (4001, 700, 4099), (4097, 200, 4090), (4001, 300, 4001), (8190, 400, 4104)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,k,n", RAGGED)
def test_linear_ragged(rows, k, n, dtype):
    """Every tile with rows and channels that end inside it: dense and pitched results, with and without a residual, nothing written
    beside them."""
    import paper_2102_08481_amd as thia
    layer, w, ws, b = layer_of(rows + n, n, k)
    codes, scales = codes_of(k, rows, k)
    out = thia.thia_linear_i8_run(layer, codes, scales, True, out_f32=dtype is F)
    check_product(out, codes, scales, w, ws, b, k, True)
    moved = torch.cat([scales[:1], scales])[1:]   # 4 bytes off
    assert torch.equal(thia.thia_linear_i8_run(layer, codes, moved, True, out_f32=dtype is F), out)
    res = rows_of(9, rows, n + 3, dtype)[:, 1:n + 1]
    want = thia.thia_linear_i8_run(layer, codes, scales, False, res.contiguous(), dtype is F)
    check_product(want, codes, scales, w, ws, b, k, False, res)
    room = torch.full((rows + 2, n + 7), 7, dtype=dtype, device="cuda")
    thia.thia_linear_i8_run(layer, codes, scales, False, res, dtype is F, out=room[:rows, 3:n + 3])
    assert torch.equal(room[:rows, 3:n + 3], want)
    room[:rows, 3:n + 3] = 7
    assert (room == 7).all()
    inplace = res.contiguous()
    thia.thia_linear_i8_run(layer, codes, scales, False, inplace, dtype is F, out=inplace)
    assert torch.equal(inplace, want)


# ragged too, with channels in eights: every tile by accesses of 16 bytes, and by single elements where the pitch is odd
RAGGED_WIDE = [(5, 200, 40), (701, 640, 136), (1003, 390, 520), (2001, 1000, 1000), (1187, 12001, 1000), (2003, 12544, 1000), (3365, 260, 1080), (2001, 200, 1992),
               (9001, 130, 1000), (2901, 300, 2008), (4001, 300, 4008), (4097, 700, 4104)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,k,n", RAGGED_WIDE)
def test_linear_ragged_by_16_bytes(rows, k, n, dtype):
    """Rows and channels that end inside the tile where rows take 16-byte accesses: dense and pitched, in place, the same bits as element by
    element, nothing written beside them."""
    import paper_2102_08481_amd as thia
    layer, w, ws, b = layer_of(rows + n, n, k)
    codes, scales = codes_of(k, rows, k)

    def pitched(columns, first):
        return torch.full((rows + 2, n + columns), 7, dtype=dtype, device="cuda")[:rows, first:first + n]

    def run(relu, res, out=None):
        return thia.thia_linear_i8_run(layer, codes, scales, relu, res, dtype is F, out)

    res = rows_of(9, rows, n, dtype) * 100
    for relu, residual in ((True, None), (False, res), (True, res)):
        want = run(relu, residual)
        check_product(want, codes, scales, w, ws, b, k, relu, residual)
        for columns, first in ((16, 8), (7, 3)):   # (the second: element by element)
            r = residual
            if r is not None:
                r = pitched(columns, first)
                r.copy_(residual)
            out = pitched(columns, first)
            room = out._base
            assert run(relu, r, out).data_ptr() == out.data_ptr() and torch.equal(out, want)
            out.fill_(7)
            assert (room == 7).all()
            if r is not None:
                assert torch.equal(run(relu, r, r), want)
                r.fill_(7)
                assert (r._base == 7).all()


def test_more_rows_than_one_launch_holds():
    import paper_2102_08481_amd as thia
    layer, w, ws, b = layer_of(3, 3, 5)
    codes, scales = codes_of(4, 1600003, 5)
    check_product(thia.thia_linear_i8_run(layer, codes, scales, out_f32=True), codes, scales, w, ws, b, 5)
    x = codes[:, :5].float()
    check_codes(*thia.thia_quantize_rows(x), x.double(), 5, 2)


@pytest.mark.parametrize("rows,k", [(33003, 65536), (270001, 8000)])
def test_offsets_beyond_32_bits(rows, k):
    """Inputs, codes and results of more than 2^31 bytes: the last rows are those of the same rows alone."""
    import paper_2102_08481_amd as thia
    x = torch.empty((rows, k), dtype=BF, device="cuda")
    x[-40:] = rows_of(1, 40, k, BF)
    x[:-40] = 1
    r = torch.zeros_like(x)
    r[-40:] = rows_of(2, 40, k, BF)
    gain = 0.5 + torch.rand(k, device="cuda")
    codes, scales = thia.thia_quantize_rows(x)
    want = thia.thia_quantize_rows(x[-40:].contiguous())
    assert torch.equal(codes[-40:], want[0]) and torch.equal(scales[-40:], want[1])
    layer, *_ = layer_of(3, 40, k)
    assert torch.equal(thia.thia_linear_i8_run(layer, codes, scales)[-40:], thia.thia_linear_i8_run(layer, *want))
    codes, scales, total = thia.thia_rms_norm_i8(x, gain, 1e-6, r)
    want = thia.thia_rms_norm_i8(x[-40:].contiguous(), gain, 1e-6, r[-40:].contiguous())
    assert all(torch.equal(a[-40:], b) for a, b in zip((codes, scales, total), want))


def test_weights_beyond_32_bits():
    """A layer of more than 2^32 bytes: its last channels are those of a layer of them alone."""
    import paper_2102_08481_amd as thia
    n, k = 70003, 65536
    w = torch.ones((n, k), dtype=torch.int8, device="cuda")
    w[-50:] = torch.randint(-127, 128, (50, k), device="cuda", dtype=torch.int8)
    one = torch.ones(n, device="cuda")
    codes, scales = codes_of(2, 37, k)
    out = thia.thia_linear_i8_run(thia.thia_linear_i8_load_codes(w, one), codes, scales)
    assert torch.equal(out[:, -50:], thia.thia_linear_i8_run(thia.thia_linear_i8_load_codes(w[-50:].contiguous(), one[:50]), codes, scales))


@pytest.mark.parametrize("n,out_f32", [(30007, True), (60000, False)])
def test_results_beyond_32_bits(n, out_f32):
    import paper_2102_08481_amd as thia
    layer, *_ = layer_of(1, n, 300)
    codes, scales = codes_of(2, 40003, 300)
    res = torch.ones((40003, n), dtype=F if out_f32 else BF, device="cuda")
    out = thia.thia_linear_i8_run(layer, codes, scales, False, res, out_f32)
    assert torch.equal(out[-70:], thia.thia_linear_i8_run(layer, codes[-70:], scales[-70:], False, res[-70:], out_f32))


@pytest.mark.parametrize("rows", [1, 20, 700, 4000])
def test_the_largest_sums(rows):
    """65536 products of -128 and -128: 2^30; and the layer takes -128 on both sides."""
    import paper_2102_08481_amd as thia
    k, n = 65536, 40
    w = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    layer = thia.thia_linear_i8_load_codes(w, torch.ones(n, device="cuda"))
    out = thia.thia_linear_i8_run(layer, torch.full((rows, k), -128, dtype=torch.int8, device="cuda"), torch.ones(rows, device="cuda"), out_f32=True)
    assert (out[:, 1] == -128.0 * 127 * k).all() and (out[:, 2:] == 2.0 ** 30).all() and (out[:, 0] == 2.0 ** 30).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_linear_with_pitches_in_place_and_beside(dtype):
    import paper_2102_08481_amd as thia
    for rows, k, n in ((5, 200, 37), (90, 200, 37), (700, 640, 130), (3000, 384, 515), (4000, 384, 512)):
        layer, w, ws, b = layer_of(n, n, k)
        codes, scales = codes_of(k, rows, k)
        room = torch.full((rows + 2, n + 7), 7, dtype=dtype, device="cuda")
        res = rows_of(9, rows, n + 3, dtype)[:, 1:n + 1]
        want = thia.thia_linear_i8_run(layer, codes, scales, False, res.contiguous(), dtype is F)
        thia.thia_linear_i8_run(layer, codes, scales, False, res, dtype is F, out=room[:rows, 3:n + 3])
        assert torch.equal(room[:rows, 3:n + 3], want)
        room[:rows, 3:n + 3] = 7
        assert (room == 7).all()   # nothing beside the rows, and nothing behind the last
        inplace = res.contiguous()
        thia.thia_linear_i8_run(layer, codes, scales, False, inplace, dtype is F, out=inplace)
        assert torch.equal(inplace, want)


def test_a_row_does_not_depend_on_the_others():
    import paper_2102_08481_amd as thia
    layer, *_ = layer_of(1, 640, 896)
    codes, scales = codes_of(2, 5000, 896)
    every = thia.thia_linear_i8_run(layer, codes, scales)
    for at, rows in ((0, 1), (17, 3), (100, 31), (500, 64), (700, 129), (1000, 300), (2000, 1000), (0, 4999)):
        assert torch.equal(thia.thia_linear_i8_run(layer, codes[at:at + rows], scales[at:at + rows]), every[at:at + rows])


@pytest.mark.parametrize("rows", [1, 50, 4000])
def test_rows_that_are_not_numbers_stay_so_and_alone(rows):
    import paper_2102_08481_amd as thia
    layer, *_ = layer_of(1, 300, 256)
    x = rows_of(4, rows, 256, BF)
    x[rows // 2, 9] = float("nan")
    codes, scales = thia.thia_quantize_rows(x)
    for relu in (False, True):
        out = thia.thia_linear_i8_run(layer, codes, scales, relu)
        bad = torch.arange(rows, device="cuda") == rows // 2
        assert out[bad].isnan().all() and not out[~bad].isnan().any()


def test_layers_from_weights_and_without_rows():
    import paper_2102_08481_amd as thia
    w = rows_of(1, 45, 333, F)
    q, s = thia.thia_quantize_rows(w)
    bias = torch.randn(45)
    codes, scales = codes_of(2, 70, 333)
    want = thia.thia_linear_i8_run(thia.thia_linear_i8_load_codes(q[:, :333], s, bias.cuda()), codes, scales)
    for weights, b in ((w, bias.cuda()), (w.cpu(), bias), (w.cpu().numpy(), bias.numpy()), (w, bias)):
        layer = thia.thia_linear_i8_load(weights, b)
        assert torch.equal(thia.thia_linear_i8_run(layer, codes, scales), want)
    assert thia.thia_linear_i8_run(layer, codes[:0], scales[:0]).shape == (0, 45)
    assert thia.thia_quantize_rows(w[:0])[0].shape == (0, 384)
    assert thia.thia_rms_norm_i8(w[:0], torch.ones(333, device="cuda"))[1].shape == (0,)
    plain = thia.thia_linear_i8_run(thia.thia_linear_i8_load(w), codes, scales, out_f32=True)
    check_product(plain, codes, scales, q[:, :333], s, torch.zeros(45, device="cuda"), 333)
    layer.close()
    with pytest.raises(thia.ThiaError):
        layer.run(codes, scales)


def test_refusals_on_the_device():
    import paper_2102_08481_amd as thia
    layer, *_ = layer_of(1, 40, 200)
    codes, scales = codes_of(2, 10, 200)
    x = rows_of(1, 10, 200, BF)
    one, cpu = torch.ones(200, device="cuda"), torch.zeros(10, 40, dtype=BF)
    for call in (lambda: layer.run(codes[:, :200], scales), lambda: layer.run(codes, scales[:9]), lambda: layer.run(codes.float(), scales), lambda: layer.run(codes.cpu(), scales),
                 lambda: layer.run(codes, scales.double()), lambda: layer.run(codes, scales, residual=cpu), lambda: layer.run(codes, scales, residual=cpu.cuda().float()),
                 lambda: layer.run(codes, scales, residual=cpu.cuda(), out_f32=True), lambda: layer.run(codes, scales, out=cpu.cuda().t().contiguous().t()),
                 lambda: layer.run(codes, scales, out=cpu.cuda()[:1].expand(10, 40)), lambda: thia.thia_quantize_rows(x.half()), lambda: thia.thia_quantize_rows(x.t()),
                 lambda: thia.thia_quantize_rows(x[0]), lambda: thia.thia_rms_norm_i8(x, one[:199]), lambda: thia.thia_rms_norm_i8(x, one.double()),
                 lambda: thia.thia_rms_norm_i8(x, one, residual=x.float()), lambda: thia.thia_rms_norm_i8(x, one, sum_out=x), lambda: thia.thia_rms_norm_i8(x, one, residual=x[:9])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: thia.thia_rms_norm_i8(x, one, 0.0), lambda: thia.thia_quantize_rows(torch.zeros(1, 65537, device="cuda")),
                 lambda: thia.thia_linear_i8_load(torch.zeros(1, 65537)), lambda: thia.thia_quantize_rows(x, out=(torch.empty(10 * 256 + 8, dtype=torch.int8, device="cuda")[8:].view(10, 256), scales))):
        with pytest.raises(thia.ThiaError):
            call()


# ---------------------------------------------------------------- together
def block(x, r, gain, up, down):
    import paper_2102_08481_amd as thia
    codes, scales, total = thia.thia_rms_norm_i8(x, gain, 1e-6, r)
    u = thia.thia_linear_i8_run(up, codes, scales, relu=True)
    c2, s2 = thia.thia_quantize_rows(u)
    return codes, scales, total, u, c2, s2, thia.thia_linear_i8_run(down, c2, s2, residual=total)


def block_parts(rows, k, n):
    import paper_2102_08481_amd as thia
    w1, w2 = rows_of(1, n, k, F) / k, rows_of(2, k, n, F) / n
    b1, b2 = torch.randn(n, device="cuda"), torch.randn(k, device="cuda")
    ups = [thia.thia_linear_i8_load(w1, b1), thia.thia_linear_i8_load(w2, b2)]
    return ups, [thia.thia_quantize_rows(w) + (b,) for w, b in ((w1, b1), (w2, b2))], 0.5 + torch.rand(k, device="cuda")


@pytest.mark.parametrize("rows,k,n", [(1, 256, 1024), (37, 200, 777), (600, 512, 1024), (4096, 256, 512)])
def test_block(rows, k, n):
    """Norm, product, codes again and product back onto the sum, as a program chains them; every step against its definition."""
    (up, down), ((q1, s1, b1), (q2, s2, b2)), gain = block_parts(rows, k, n)
    x, r = rows_of(3, rows, k, BF), rows_of(4, rows, k, BF)
    codes, scales, total, u, c2, sc2, out = block(x, r, gain, up, down)
    h = (x.float() + r.float()).double()
    check_codes(codes, scales, h * gain.double() / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6), k, 64)
    check_product(u, codes, scales, q1[:, :k], s1, b1, k, True)
    check_codes(c2, sc2, u.double(), n, 2)
    check_product(out, c2, sc2, q2[:, :n], s2, b2, n, False, total)


def test_block_captured_and_on_other_streams():
    """A captured chain gives the eager results at every replay, on changing inputs and with eager work in between; chains of the
    same layers on two streams at once do too."""
    (up, down), _, gain = block_parts(300, 512, 1024)
    x, r = rows_of(3, 300, 512, BF), rows_of(4, 300, 512, BF)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(x, r, gain, up, down)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = block(x, r, gain, up, down)
    for seed in range(4):
        x.copy_(rows_of(10 + seed, 300, 512, BF))
        graph.replay()
        want = block(x, r, gain, up, down)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
    ys, others = [rows_of(20 + i, 300, 512, BF) for i in range(6)], [torch.cuda.Stream() for _ in range(2)]
    want = [block(y, r, gain, up, down)[-1] for y in ys]
    torch.cuda.synchronize()
    got = []
    for i, y in enumerate(ys):
        with torch.cuda.stream(others[i % 2]):
            got.append(block(y, r, gain, up, down)[-1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_threads_at_once():
    """Calls from two threads, each on a stream of its own, with one layer: nothing is shared between calls."""
    import threading
    (up, down), _, gain = block_parts(300, 512, 1024)
    r = rows_of(4, 300, 512, BF)
    xs = [rows_of(30 + i, 300, 512, BF) for i in range(2)]
    want = [block(x, r, gain, up, down)[-1] for x in xs]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got[i].append(block(xs[i], r, gain, up, down)[-1])
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(len(g) == 20 and all(torch.equal(v, w) for v in g) for g, w in zip(got, want))


# ---------------------------------------------------------------- the box head in 8 bits
def head_layers(spec, blob, ep):
    """Exit ep's wide layers from the blob, in the element type and order the library keeps them, and the predictors in 64 bits."""
    import paper_2102_08481_amd as thia
    from thia_synth import split_blob
    t = {k: torch.from_numpy(v.copy()).cuda() for k, v in split_blob(spec, blob).items() if k.startswith(f"e{ep}.")}
    dtype = BF if spec.precision else F
    w1 = t[f"e{ep}.fc1.w"]
    w1 = w1.reshape(w1.shape[0], -1, 49).transpose(1, 2).reshape(w1.shape[0], -1)   # [c][bin] -> [bin][c]
    layers = [thia.thia_linear_i8_load(w.to(dtype).float(), t[f"e{ep}.{n}.b"]) for n, w in (("fc1", w1), ("fc2", t[f"e{ep}.fc2.w"]))]
    return layers, [(t[f"e{ep}.{n}.w"].to(dtype).double(), t[f"e{ep}.{n}.b"].double()) for n in ("cls", "box")]


@pytest.mark.parametrize("precision,head_ch", [(1, 256), (0, 256), (1, 64)])
def test_box_head_in_8_bits(precision, head_ch):
    """The head's wide layers in 8 bits are the public calls on the same rows, bit for bit; back in the model's type everything is as
    it was; frames do not depend on their neighbours.  Without taps, five frames' regions become codes in ROIAlign itself, one frame's behind it:
    the same."""
    from dataclasses import replace
    import numpy as np
    import paper_2102_08481_amd as thia
    from gpu_common import MINI_BF16, MINI_FP32, biased_model
    spec = replace(MINI_BF16 if precision else MINI_FP32, head_ch=head_ch, post_nms=300)
    model, blob = biased_model(spec, 77)
    frames = torch.from_numpy(np.random.RandomState(5).randint(0, 256, (5, 3, 130, 190)).astype(np.uint8)).cuda()
    ep = 2
    before = [v.clone() for v in model.detect_chunk(frames, ep)]
    try:
        model.set_head_bits(8)
        model.set_debug(True)
        eight = [v.clone() for v in model.detect_chunk(frames, ep)]
        torch.cuda.synchronize()
        feat = torch.from_numpy(model.tap("roi_feat")).cuda().to(BF if precision else F).reshape(5 * spec.post_nms, -1)
        logits, deltas = (torch.from_numpy(model.tap(n)).cuda().double().reshape(5 * spec.post_nms, -1) for n in ("cls_logits", "box_deltas"))
        model.set_debug(False)
        (fc1, fc2), preds = head_layers(spec, blob, ep)
        h1 = thia.thia_linear_i8_run(fc1, *thia.thia_quantize_rows(feat), relu=True, out_f32=not precision)
        h2 = thia.thia_linear_i8_run(fc2, *thia.thia_quantize_rows(h1), relu=True, out_f32=not precision).double()
        for got, (w, b) in zip((logits, deltas), preds):
            # products of the same elements added in fp32, `fc_dim` of them and the bias, each addition off by at most 1 u of the sum of sizes
            size = h2.abs() @ w.abs().t().contiguous() + b.abs()
            assert ((got - (h2 @ w.t().contiguous() + b)).abs() <= (spec.fc_dim + 2) * U * size).all()
        for i in range(5):
            alone = model.detect_chunk(frames[i:i + 1].contiguous(), ep)
            assert all(torch.equal(a[0], b[i]) for a, b in zip(alone, eight))
        chunks = model.run_chunks(frames, [(0, 2, ep), (2, 3, ep)])
        assert all(torch.equal(a, b) for a, b in zip(chunks, eight))
        every = model.detect_all_exits(frames)
        assert all(torch.equal(a[ep - 1], b) for a, b in zip(every, eight))
        with pytest.raises(thia.ThiaError):
            model.set_head_bits(4)
    finally:
        model.set_debug(False)
        model.set_head_bits(0)
    assert all(torch.equal(a, b) for a, b in zip(before, model.detect_chunk(frames, ep)))
    assert not torch.equal(before[1], eight[1])   # the option does something


@pytest.mark.parametrize("precision", [1, 0])
def test_how_far_the_head_in_8_bits_is_from_the_models_own(precision):
    """Logits and deltas of the two heads on the same region features.  A code is off by at most half a step of its row, step / sqrt(12) in the
    mean square if what is rounded off is spread evenly, and those errors are independent of one another: their squares add up along the
    products, through both layers and the predictors, as do those of the results' rounding to bf16.  They would have to double for errors
    of half a step each (sqrt(3) of the even spread); twice the predicted deviation holds for each exit's logits and deltas taken together."""
    import numpy as np
    from gpu_common import MINI_BF16, MINI_FP32, biased_model
    from thia_synth import split_blob
    spec = MINI_BF16 if precision else MINI_FP32
    model, blob = biased_model(spec, 77)
    frames = torch.from_numpy(np.random.RandomState(6).randint(0, 256, (2, 3, 130, 190)).astype(np.uint8)).cuda()
    dtype, rows = BF if precision else F, 2 * spec.post_nms
    for ep in (1, spec.n_exits):
        t = {n: torch.from_numpy(v.copy()).cuda() for n, v in split_blob(spec, blob).items() if n.startswith(f"e{ep}.")}
        w = {n: t[f"e{ep}.{n}.w"].to(dtype).double() for n in ("fc1", "fc2", "cls", "box")}
        w["fc1"] = w["fc1"].reshape(spec.fc_dim, -1, 49).transpose(1, 2).reshape(spec.fc_dim, -1)
        taps = {}
        try:
            model.set_debug(True)
            for bits in (0, 8):
                model.set_head_bits(bits)
                model.detect_chunk(frames, ep)
                torch.cuda.synchronize()
                taps[bits] = {n: torch.from_numpy(model.tap(n).copy()).cuda().double().reshape(rows, -1) for n in ("roi_feat", "cls_logits", "box_deltas")}
        finally:
            model.set_debug(False)
            model.set_head_bits(0)
        assert torch.equal(taps[0]["roi_feat"], taps[8]["roi_feat"])
        h, var = taps[0]["roi_feat"], 0.0
        for n in ("fc1", "fc2"):
            a, b = h.abs().amax(1, keepdim=True) / 127, w[n].abs().amax(1) / 127   # the steps
            wt = w[n].t().contiguous()
            var = (var + (h != 0) * a * a / 12) @ (wt * wt) + (h * h) @ ((wt != 0) * b * b / 12)
            h = (h @ wt + t[f"e{ep}.{n}.b"].double()).clamp(min=0)
            var = var * (h > 0) + (2 * (h * HALF[dtype]) ** 2 / 3 if precision else 0)
        for name, n in (("cls_logits", "cls"), ("box_deltas", "box")):
            wt = w[n].t().contiguous()
            off = taps[8][name] - taps[0][name]
            got, predicted = (off * off).mean().sqrt(), (var @ (wt * wt)).mean().sqrt()
            assert 0 < got <= 2 * predicted


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_head_bits_belong_to_the_models_device():
    """The 8-bit layers are refused while another device is current, and the model stays as it was."""
    import numpy as np
    import paper_2102_08481_amd as thia
    from gpu_common import MINI_BF16, biased_model
    model, _ = biased_model(MINI_BF16, 77)
    frames = torch.from_numpy(np.random.RandomState(5).randint(0, 256, (1, 3, 130, 190)).astype(np.uint8)).cuda()
    before = [v.clone() for v in model.detect_chunk(frames, 1)]
    with torch.cuda.device(1), pytest.raises(thia.ThiaError):
        model.set_head_bits(8)
    assert all(torch.equal(a, b) for a, b in zip(before, model.detect_chunk(frames, 1)))
