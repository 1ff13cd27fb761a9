"""Rows of 4-bit floats with a scale for every 32 dimensions: quantisation and its way back, cosine inference, products and online
training on such rows, against the oracle in 64 bits.  Sizes on both sides of a block of 32 dimensions, of a wave's and a block's rows,
single samples and rows; rows of zeros, of the ends of fp32's range, with infinities and what is no number; scales that lie far apart;
other streams, replays of a graph, labels outside the range."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import quantized as oq  # noqa: E402
from workloads import make_workload  # noqa: E402

from test_gpu_parity import dev_u32, make_ctx  # noqa: E402

U = 2.0 ** -53


def context(D, C=2):
    return make_ctx(make_workload(1, D=D, C=C, F=3, L=2))


def words(rng, N, D):
    hv = rng.integers(0, 1 << 32, (N, (D + 31) // 32), dtype=np.uint32)
    if D % 32:
        hv[:, -1] &= np.uint32((1 << (D % 32)) - 1)
    return hv


def rows_of(kind, N, D, rng):
    x = rng.normal(size=(N, D))
    if kind == "orders":          # elements and blocks of very different sizes
        x *= np.exp(6 * rng.normal(size=(N, D)))
    if kind == "steps":           # the values between which the rounding changes, and their neighbours, at scales of all kinds
        x = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.5, 1.0, 0.0], size=(N, D)) * rng.choice([-1, 1], size=(N, D))
        x = np.nextafter(x.astype(np.float32), rng.choice([-np.inf, 0, np.inf], size=(N, D)).astype(np.float32)) if rng.random() < 0.5 else x
        x = x * np.exp2(np.repeat(rng.integers(-150, 126, size=(N, (D + 31) // 32)), 32, axis=1)[:, :D].astype(np.float64))
    if kind == "tiny":
        x = x * 2.0 ** -126 * np.exp2(-rng.integers(0, 24, size=(N, D)).astype(np.float64))
    if kind == "zeros":
        x *= np.repeat(rng.random((N, (D + 31) // 32)) < 0.3, 32, axis=1)[:, :D] * np.where(rng.random((N, D)) < 0.5, -1, 1)
    with np.errstate(over="ignore", under="ignore"):
        x = np.clip(x, -3.4e38, 3.4e38).astype(np.float32)
    if kind == "none":            # some infinite, some no numbers
        x[rng.random((N, D)) < 0.01] = np.nan
        x[rng.random((N, D)) < 0.01] = -np.inf
        x[0, -1] = np.inf
    return x


def quantized(x, ctx=None, norm=True):
    """What the library makes of rows, on the device."""
    N, D = x.shape
    own = ctx or context(D)
    W = (D + 31) // 32
    codes = torch.full((N, 4 * W), -1, dtype=torch.int32, device="cuda")
    scales = torch.full((N, W), 77, dtype=torch.uint8, device="cuda")
    norms = torch.full((N,), -1.0, dtype=torch.float64, device="cuda") if norm else None
    own.hdc_quantize(torch.from_numpy(x).cuda(), codes, scales, norms)
    torch.cuda.synchronize()
    if ctx is None:
        own.close()
    return codes, scales, norms


def same_bits(a, b):
    """Equal numbers of equal signs (zeros too); what is no number in both."""
    return np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(a)].view(np.uint32), b[~np.isnan(b)].view(np.uint32))


KINDS = ["normal", "orders", "steps", "tiny", "zeros", "none"]


# ---- quantisation: codes and scales have no rounding of their own but the one defined; a norm is a sum of W terms or fewer
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,D", [(1, 1), (3, 31), (2, 32), (5, 33), (7, 63), (4, 64), (9, 65), (130, 100), (2, 127), (3, 500), (6, 1024), (1, 4097),
                                 (6, 10000), (300, 1021), (2, 40003), (70001, 5)])
def test_rows_become_the_defined_codes(kind, N, D):
    x = rows_of(kind, N, D, np.random.default_rng(N * 7 + D))
    codes, scales, norm = quantized(x)
    W = (D + 31) // 32
    want_codes, want_scales, v, want_norm = oq.quantize(x)
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy().view(np.uint32), want_codes)
    got = norm.cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want_norm))
    ok = ~np.isnan(want_norm)
    assert np.all(np.abs(got - want_norm)[ok] <= (2 * W + 70) * U * want_norm[ok])     # (numpy's own sum among it)
    # and back
    ctx = context(D)
    back = torch.full((N, D), 5.0, dtype=torch.float32, device="cuda")
    ctx.hdc_dequantize(codes, scales, back)
    torch.cuda.synchronize()
    ctx.close()
    assert same_bits(back.cpu().numpy(), v.astype(np.float32))


def test_rows_of_the_largest_dimension_and_rows_without_norms():
    rng = np.random.default_rng(1)
    x = rows_of("orders", 3, 1048576 - 5, rng)
    codes, scales, norm = quantized(x)
    want_codes, want_scales, v, want_norm = oq.quantize(x)
    assert np.array_equal(scales.cpu().numpy(), want_scales) and np.array_equal(codes.cpu().numpy().view(np.uint32), want_codes)
    assert np.all(np.abs(norm.cpu().numpy() - want_norm) <= 70000 * U * want_norm)
    again, scales_again, none = quantized(x, norm=False)
    assert none is None and torch.equal(again, codes) and torch.equal(scales_again, scales)


def test_neighbours_of_the_rows_are_left_alone():
    """Rows written into the middle of larger arrays, from the middle of others (rows of 33 dimensions start anywhere)."""
    rng = np.random.default_rng(2)
    D, W = 33, 2
    x = rows_of("normal", 12, D, rng)
    ctx = context(D)
    big = torch.from_numpy(x).cuda()
    codes = torch.full((12, 4 * W), -1, dtype=torch.int32, device="cuda")
    scales = torch.full((12, W), 77, dtype=torch.uint8, device="cuda")
    norm = torch.full((12,), -1.0, dtype=torch.float64, device="cuda")
    ctx.hdc_quantize(big[3:8], codes[3:8], scales[3:8], norm[3:8])
    back = torch.full((12, D), 9.0, device="cuda")
    ctx.hdc_dequantize(codes[3:8], scales[3:8], back[3:8])
    torch.cuda.synchronize()
    want_codes, want_scales, v, _ = oq.quantize(x)
    inside = np.arange(12) // 1
    inside = (inside >= 3) & (inside < 8)
    assert np.array_equal(codes.cpu().numpy().view(np.uint32)[inside], want_codes[inside]) and np.all(codes.cpu().numpy()[~inside] == -1)
    assert np.array_equal(scales.cpu().numpy()[inside], want_scales[inside]) and np.all(scales.cpu().numpy()[~inside] == 77)
    assert np.all(norm.cpu().numpy()[~inside] == -1) and np.all(back.cpu().numpy()[~inside] == 9)
    assert same_bits(back.cpu().numpy()[inside], v.astype(np.float32)[inside])
    ctx.close()


@pytest.mark.parametrize("D", [1, 3, 29, 64, 257, 1000, 2055])
def test_rows_written_from_any_place(D):
    """Rows that start anywhere in a cache line, with blocks that are no numbers and the bits beyond D set; what is around them is left alone."""
    rng = np.random.default_rng(D)
    N, W = 41, (D + 31) // 32
    codes = rng.integers(0, 2 ** 32, size=(N, 4 * W), dtype=np.uint32)
    scales = rng.choice(np.array([0, 1, 100, 127, 128, 140, 252, 255], np.uint8), size=(N, W))
    with np.errstate(over="ignore"):
        want = oq.values(codes, scales, D).astype(np.float32)
    ctx = context(D)
    c, s = dev_u32(codes), torch.from_numpy(scales).cuda()
    for start in (0, 1, 2, 3, 4, 5, 7, 12, 30, 31, 33):
        room = torch.full((start + N * D + 40,), 9.0, device="cuda")
        ctx.hdc_dequantize(c, s, room[start:start + N * D].view(N, D))
        torch.cuda.synchronize()
        got = room.cpu().numpy()
        assert same_bits(got[start:start + N * D].reshape(N, D), want)
        assert np.all(got[:start] == 9) and np.all(got[start + N * D:] == 9)
    ctx.close()


def test_scales_that_quantisation_does_not_give():
    """s = 253 and 254: values beyond fp32 are infinite; every code at every scale."""
    D = 512
    codes = np.tile(np.array([sum(((i * 4 + r) % 16) << 4 * i for i in range(8)) for r in range(4)], np.uint64).astype(np.uint32), (256, 16))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, axis=1)
    ctx = context(D)
    back = torch.empty((256, D), device="cuda")
    ctx.hdc_dequantize(dev_u32(codes), torch.from_numpy(scales).cuda(), back)
    torch.cuda.synchronize()
    ctx.close()
    with np.errstate(over="ignore"):
        assert same_bits(back.cpu().numpy(), oq.values(codes, scales, D).astype(np.float32))


# ---- inference: a dot product is without rounding or a sum of W whole numbers in fp64, so a cosine, at most 1, is off by W + 8 roundings
# of 2^-53 and the one to fp32
def check_search(hv, x, codes=None, scales=None, want_cos=True, tie_ok=True):
    N, (C, D) = hv.shape[0], x.shape
    W = (D + 31) // 32
    ctx = context(D, C)
    if codes is None:
        codes, scales, norm = quantized(x, ctx)
    else:
        v = oq.values(codes, scales, D)
        codes, scales, norm = dev_u32(codes), torch.from_numpy(scales).cuda(), torch.from_numpy((v * v).sum(1)).cuda()
    pred = torch.full((N,), -7, dtype=torch.int32, device="cuda")
    cos = torch.full((N, C), 7.0, dtype=torch.float32, device="cuda") if want_cos else None
    ctx.hdc_search_quantized(dev_u32(hv), codes, scales, norm, pred, cos)
    torch.cuda.synchronize()
    ctx.close()
    want = oq.cosines(hv, oq.values(codes.cpu().numpy(), scales.cpu().numpy(), D), norm.cpu().numpy())
    slack = (W + 8) * U
    pred = pred.cpu().numpy()
    if want_cos:
        got = cos.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        assert np.all(np.abs(got - want)[ok] <= 2.0 ** -24 * np.abs(want)[ok] * (1 + 1e-6) + 1.5 * slack)
    assert pred.min() >= 0 and pred.max() < C
    for n in np.flatnonzero(np.isnan(want).all(1)):
        assert pred[n] == 0
    number = ~np.isnan(want).all(1)
    best = np.nanmax(want[number], axis=1) if number.any() else np.zeros(0)
    mine = want[number, pred[number]]
    assert np.all(mine >= best - 3 * slack)
    clear = np.sort(np.where(np.isnan(want), -2, want), axis=1)
    clear = clear[:, -1] - (clear[:, -2] if C > 1 else -2) > 3 * slack
    assert np.array_equal(pred[clear], oq.nearest(want)[clear])
    return pred, want


SEARCH = [(1, 1, 1), (1, 6, 10000), (2, 2, 31), (15, 5, 33), (16, 16, 128), (17, 17, 129), (33, 26, 1000), (64, 3, 4096), (65, 1, 4097), (100, 64, 500),
          (127, 33, 2047), (129, 100, 777), (300, 6, 10000), (513, 26, 1024), (1100, 10, 3001), (4, 1024, 1000), (40, 1000, 4099), (2, 300, 16385),
          (3, 9, 70001), (5000, 2, 96), (2947, 6, 2500)]


@pytest.mark.parametrize("kind", ["normal", "orders", "zeros", "none", "tiny"])
@pytest.mark.parametrize("N,C,D", SEARCH)
def test_cosines_with_quantised_rows(N, C, D, kind):
    rng = np.random.default_rng(N + C * 3 + D * 11)
    x = rows_of(kind, C, D, rng)
    if kind == "zeros" and C > 2:
        x[C // 2] = 0
    check_search(words(rng, N, D), x, want_cos=N % 2 == 1 or C < 7)


# many samples and classes: tiles of 128 classes and 256 samples, with some past their ends
MANY = [(16500, 65, 500), (8200, 129, 300), (9000, 200, 1021), (3000, 1000, 257), (2049, 1024, 2081), (33000, 64, 225),
        (25000, 65, 500), (12545, 129, 300), (13000, 200, 1021), (3100, 1024, 2081), (24577, 128, 4097), (33000, 1024, 290), (26000, 100, 200)]


@pytest.mark.parametrize("kind", ["normal", "zeros", "none", "orders"])
@pytest.mark.parametrize("N,C,D", MANY)
def test_cosines_of_many_samples_with_many_rows(N, C, D, kind):
    rng = np.random.default_rng(N + C * 3 + D * 11)
    x = rows_of("normal" if kind == "none" else kind, C, D, rng)
    if kind == "none":
        x[3, D // 2], x[C - 1, 0] = np.nan, np.inf
    if kind == "zeros":
        x[C // 2] = 0
    check_search(words(rng, N, D), x, want_cos=N != 3000)


# very many samples of short rows: a row to one wave, two or four
SHORT = [(50000, 3, 96), (50001, 10, 97), (49999, 26, 500), (50000, 16, 1025), (60001, 26, 700), (50017, 9, 2048), (50000, 20, 1500), (49200, 5, 3001),
         (49160, 26, 2500), (50000, 40, 600), (66000, 64, 1000), (49153, 6, 4500)]


@pytest.mark.parametrize("kind", ["normal", "zeros", "none", "orders"])
@pytest.mark.parametrize("N,C,D", SHORT)
def test_cosines_of_many_samples_with_short_rows(N, C, D, kind):
    rng = np.random.default_rng(N + C * 3 + D * 11)
    x = rows_of("normal" if kind == "none" else kind, C, D, rng)
    if kind == "none":
        x[1, D // 2], x[C - 1, 0] = np.nan, np.inf
    if kind == "zeros":
        x[C // 2] = 0
    check_search(words(rng, N, D), x, want_cos=kind in ("none", "orders"))
    if kind == "orders":
        check_search(words(rng, N, D), x, want_cos=False)


@pytest.mark.parametrize("N,C", [(17000, 70), (25000, 70), (8200, 300), (50000, 30), (50000, 14)])
def test_equal_cosines_of_many_samples_go_to_the_lowest_class(N, C):
    """Rows that repeat, within a tile of classes and across, and multiples of one another by powers of two."""
    rng = np.random.default_rng(C)
    D = 400
    x = rows_of("normal", C, D, rng)
    x[9:] = x[rng.integers(0, 9, C - 9)] * np.exp2(rng.integers(-6, 7, C - 9))[:, None]
    pred, want = check_search(words(rng, N, D), x.astype(np.float32))
    assert np.all(pred < 9) and np.array_equal(pred, want[:, :9].argmax(1))


def test_equal_cosines_go_to_the_lowest_class():
    """Rows that repeat, and rows that are multiples of one another by powers of two."""
    rng = np.random.default_rng(5)
    N, C, D = 70, 40, 1000
    x = rows_of("normal", C, D, rng)
    x[7:] = x[rng.integers(0, 7, C - 7)] * np.exp2(rng.integers(-6, 7, C - 7))[:, None]
    hv = words(rng, N, D)
    codes, scales, v, norm = oq.quantize(x.astype(np.float32))
    pred, want = check_search(hv, x.astype(np.float32))
    assert np.all(pred < 7) and np.array_equal(pred, want[:, :7].argmax(1))


@pytest.mark.parametrize("N,C,D", [(3, 2, 100), (50, 20, 5000), (600, 6, 10000), (20, 70, 3001)])
def test_scales_far_apart_are_summed_without_loss(N, C, D):
    """Blocks whose scales differ by up to 2^60 cancel but for the smallest: exact sums tell the classes apart."""
    rng = np.random.default_rng(D)
    W = (D + 31) // 32
    codes = rng.integers(0, 1 << 32, (C, 4 * W), dtype=np.uint64).astype(np.uint32)
    if D % 32:
        for i in range(D % 32, 32):
            codes[:, 4 * (W - 1) + i % 4] &= np.uint32(~(0xF << 4 * (i // 4)) & 0xFFFFFFFF)
    scales = rng.integers(97, 158, (C, W)).astype(np.uint8)
    check_search(words(rng, N, D), np.zeros((C, D)), codes, scales)


# ---- products: fp32 sums of D terms; without rounding where the sums fit 24 bits
def check_product(xa, xb):
    (M, D), N = xa.shape, xb.shape[0]
    ctx = context(D)
    a, sa, _ = quantized(xa, ctx, norm=False)
    b, sb, _ = quantized(xb, ctx, norm=False)
    out = torch.full((M + 2, N), 3.0, dtype=torch.float32, device="cuda")
    ctx.hdc_product_quantized(a, sa, b, sb, out[1:M + 1])
    torch.cuda.synchronize()
    ctx.close()
    va, vb = oq.values(a.cpu().numpy(), sa.cpu().numpy(), D), oq.values(b.cpu().numpy(), sb.cpu().numpy(), D)
    got = out.cpu().numpy()
    assert np.all(got[0] == 3) and np.all(got[-1] == 3)
    with np.errstate(invalid="ignore"):
        return got[1:-1].astype(np.float64), va @ vb.T, np.abs(va) @ np.abs(vb).T


PRODUCT = [(1, 1, 1), (1, 26, 10000), (26, 1, 10000), (2, 3, 31), (16, 16, 128), (17, 15, 129), (32, 33, 64), (33, 31, 65), (100, 26, 500), (64, 130, 1000),
           (129, 257, 777), (300, 200, 3001), (1, 1000, 1024), (700, 2, 4097), (5, 7, 70001), (255, 513, 96), (400, 300, 3001), (515, 1030, 512), (600, 600, 513), (700, 650, 545), (1000, 700, 1000),
           (1290, 1300, 769), (513, 600, 2100), (1500, 1500, 801)]


@pytest.mark.parametrize("kind", ["normal", "orders", "zeros", "tiny"])
@pytest.mark.parametrize("M,N,D", PRODUCT)
def test_products_of_quantised_rows(M, N, D, kind):
    rng = np.random.default_rng(M + N * 3 + D * 11)
    # (tiny rows with large ones: the product of two blocks below 2^-126 is below what fp32 holds)
    xa, xb = rows_of(kind, M, D, rng), rows_of(kind, N, D, rng) if kind != "tiny" else (rows_of("normal", N, D, rng) * 2.0 ** 60).astype(np.float32)
    got, want, size = check_product(xa, xb)
    if kind == "normal" and D <= 4097:
        # scales of a block lie between 2^-3 and 2^0 (largest of 32 normal values), so that products are whole multiples of 2^-8 (2^-2 of
        # the codes, 2^-6 of the scales) and sums of magnitudes below 2^16 fit 24 bits
        exact = size < 2 ** 16
        few = np.array([min(oq.quantize(xa)[1].min(), oq.quantize(xb)[1].min())])
        if D % 32 == 0 and few[0] >= 124:
            assert np.array_equal(got[exact], want[exact])
    assert np.all(np.abs(got - want) <= (D + 2) * 2.0 ** -24 * size)


# tiles of 128 and of 256 rows through LDS, with rows and dimensions past their ends
@pytest.mark.parametrize("M,N,D", [(1100, 1000, 33), (1025, 1030, 1000), (900, 2100, 256), (4200, 4000, 250), (4097, 4097, 31), (3900, 4300, 2081), (64, 33000, 512)])
def test_products_of_many_rows(M, N, D):
    rng = np.random.default_rng(M + N * 3 + D * 11)
    xa, xb = rows_of("normal", M, D, rng), rows_of("normal", N, D, rng)
    xa[M // 2, D // 2] = np.nan
    got, want, size = check_product(xa, xb)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.all(np.abs(got - want)[ok] <= (D + 2) * 2.0 ** -24 * size[ok])


def test_products_with_blocks_that_are_no_number():
    rng = np.random.default_rng(8)
    got, want, _ = check_product(rows_of("none", 40, 300, rng), rows_of("none", 50, 300, rng))
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).any()
    rng = np.random.default_rng(9)
    xa, xb = rows_of("normal", 40, 300, rng), rows_of("normal", 50, 300, rng)
    xa[7, 100] = np.nan
    xb[9, 299] = np.inf
    got, want, size = check_product(xa, xb)
    assert np.isnan(got[7]).all() and np.isnan(got[:, 9]).all() and np.isnan(got).sum() == 40 + 50 - 1
    ok = ~np.isnan(want)
    assert np.all(np.abs(got - want)[ok] <= 302 * 2.0 ** -24 * size[ok])


# ---- training: one batch from given rows.  A weight may be rounded the other way (2^-24 of it, at most 2: 2^-23 each of those that a row
# took), then the element is rounded to fp32
def run_training(hv, y, acc, batch, epochs, lr, reserve=True):
    C, D = acc.shape
    W = (D + 31) // 32
    ctx = context(D, C)
    rows = torch.from_numpy(acc.copy()).cuda()
    codes = torch.full((C, 4 * W), -1, dtype=torch.int32, device="cuda")
    scales = torch.full((C, W), 7, dtype=torch.uint8, device="cuda")
    norm = torch.full((C,), -1.0, dtype=torch.float64, device="cuda")
    ctx.hdc_train_online_quantized(dev_u32(hv), torch.from_numpy(y).cuda(), rows, codes, scales, norm, batch, epochs, lr)
    torch.cuda.synchronize()
    ctx.close()
    return rows.cpu().numpy(), codes.cpu().numpy().view(np.uint32), scales.cpu().numpy(), norm.cpu().numpy()


def check_batch(hv, y, acc, lr):
    got, codes, scales, norm = run_training(hv, y, acc, len(y), 1, lr)
    want, weights = oq.train_batch(hv, y, acc, lr)
    assert np.all(np.abs(got.astype(np.float64) - want) <= 2.0 ** -24 * np.abs(want) * 2 + 2.0 ** -23 * weights[:, None])
    # what is left is the quantisation of the rows that are left
    want_codes, want_scales, _, want_norm = oq.quantize(got)
    assert np.array_equal(codes, want_codes) and np.array_equal(scales, want_scales)
    assert np.allclose(norm, want_norm, rtol=1e-12, atol=0)


TRAIN = [(1, 1, 1), (3, 2, 31), (40, 5, 100), (64, 6, 1024), (100, 26, 500), (33, 40, 300), (1500, 20, 200), (2100, 6, 130), (500, 300, 96), (7, 3, 10000), (20000, 6, 130), (20000, 26, 97)]


@pytest.mark.parametrize("start", ["zeros", "sums"])
@pytest.mark.parametrize("N,C,D", TRAIN)
def test_one_batch_of_training(N, C, D, start):
    rng = np.random.default_rng(N + C + D)
    hv = words(rng, N, D)
    y = rng.integers(-1, C + 1, N).astype(np.int32)     # outside [0, C): skipped
    acc = np.zeros((C, D), np.float32)
    if start == "sums":
        acc = np.rint(30 * rng.normal(size=(C, D))).astype(np.float32)
    check_batch(hv, y, acc, 0.7)


@pytest.mark.parametrize("kind", ["normal", "orders"])
@pytest.mark.parametrize("C", [7, 20, 40])
@pytest.mark.parametrize("D", [2048, 2049, 4097, 6145, 8193, 10241, 12289, 14337, 16385, 20481])
def test_every_length_of_rows(D, C, kind):
    """Lengths around which more of a row is held at a time, and those that go in parts: searched and trained."""
    rng = np.random.default_rng(D + C)
    x = rows_of(kind, C, D, rng)
    check_search(words(rng, 37, D), x)
    check_batch(words(rng, 70, D), rng.integers(0, C, 70).astype(np.int32), x if kind == "normal" else np.clip(x, -1e6, 1e6), 0.5)


@pytest.mark.parametrize("N,C,D", [(60, 6, 300), (60, 20, 300), (1200, 20, 300), (60, 40, 300)])
def test_training_with_rows_that_are_no_numbers(N, C, D):
    """Such a row is never predicted, its own samples make all of it no numbers, the others are trained as ever; of all such rows none is predicted."""
    rng = np.random.default_rng(N + C)
    hv, y = words(rng, N, D), rng.integers(0, C, N).astype(np.int32)
    acc = np.rint(10 * rng.normal(size=(C, D))).astype(np.float32)
    acc[1, 40], acc[2, 299] = np.inf, np.nan
    got, codes, scales, norm = run_training(hv, y, acc, N, 1, 0.7)
    want, weights = oq.train_batch(hv, y, acc, 0.7)
    # (a class without samples keeps its row)
    assert all(np.isnan(got[c]).all() if np.any(y == c) else np.array_equal(got[c], acc[c], equal_nan=True) for c in (1, 2))
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = np.arange(C) != 1
    fine[2] = False
    assert np.all(np.abs(got[fine].astype(np.float64) - want[fine]) <= 2.0 ** -24 * np.abs(want[fine]) * 2 + 2.0 ** -23 * weights[fine, None])
    want_codes, want_scales, _, _ = oq.quantize(got)
    assert np.array_equal(codes, want_codes) and np.array_equal(scales, want_scales) and np.isnan(norm[1:3]).all() and np.isfinite(norm[fine]).all()
    acc[:, 7] = np.inf
    got = run_training(hv, np.where(y == 3, 4, y).astype(np.int32), acc, N, 1, 0.7)[0]
    with np.errstate(invalid="ignore"):
        assert np.array_equal(got[3], acc[3])       # nothing was added, nothing taken away


def test_training_without_norms():
    rng = np.random.default_rng(8)
    N, C, D = 90, 6, 300
    hv, y = words(rng, N, D), rng.integers(0, C, N).astype(np.int32)
    acc = np.rint(10 * rng.normal(size=(C, D))).astype(np.float32)
    want = run_training(hv, y, acc, 32, 2, 1.0)
    ctx = context(D, C)
    rows = torch.from_numpy(acc.copy()).cuda()
    codes, scales = torch.zeros((C, 40), dtype=torch.int32, device="cuda"), torch.zeros((C, 10), dtype=torch.uint8, device="cuda")
    ctx.hdc_train_online_quantized(dev_u32(hv), torch.from_numpy(y).cuda(), rows, codes, scales, None, 32, 2, 1.0)
    torch.cuda.synchronize()
    ctx.close()
    assert np.array_equal(rows.cpu().numpy(), want[0]) and np.array_equal(codes.cpu().numpy().view(np.uint32), want[1])
    assert np.array_equal(scales.cpu().numpy(), want[2])


@pytest.mark.parametrize("N,C,D,batch,epochs", [(50, 3, 200, 16, 2), (300, 26, 333, 64, 1), (70, 2, 64, 1, 1)])
def test_batches_follow_one_another(N, C, D, batch, epochs):
    """A call is its batches, one call each."""
    rng = np.random.default_rng(N)
    hv, y = words(rng, N, D), rng.integers(0, C, N).astype(np.int32)
    acc = np.rint(10 * rng.normal(size=(C, D))).astype(np.float32)
    got = run_training(hv, y, acc, batch, epochs, 1.0)
    for _ in range(epochs):
        for n in range(0, N, batch):
            step = run_training(hv[n:n + batch], y[n:n + batch], acc, batch, 1, 1.0)
            acc = step[0]
    for a, b in zip(got, step):
        assert np.array_equal(a, b)


def test_training_refuses_bad_labels_when_asked_and_leaves_everything():
    from paper_2206_04746_amd import binding
    rng = np.random.default_rng(3)
    ctx = context(100, 4)
    ctx.hdc_set_label_check(True)
    acc, codes = torch.ones((4, 100), device="cuda"), torch.full((4, 16), 3, dtype=torch.int32, device="cuda")
    scales, norm = torch.full((4, 4), 3, dtype=torch.uint8, device="cuda"), torch.full((4,), 3.0, dtype=torch.float64, device="cuda")
    hv, y = dev_u32(words(rng, 5, 100)), torch.tensor([0, 1, 4, 2, 3], dtype=torch.int32, device="cuda")
    with pytest.raises(binding.HdcError) as e:
        ctx.hdc_train_online_quantized(hv, y, acc, codes, scales, norm, 2)
    assert e.value.code == binding.HDC_ELABEL
    ctx.hdc_train_online_quantized(hv[:0], y[:0], acc, codes, scales, norm, 2)
    ctx.hdc_train_online_quantized(hv, torch.zeros_like(y), acc, codes, scales, norm, 2, epochs=0)
    torch.cuda.synchronize()
    assert bool((acc == 1).all()) and bool((codes == 3).all()) and bool((scales == 3).all()) and bool((norm == 3).all())
    ctx.close()


def test_binding_refuses_other_shapes_and_types():
    ctx = context(100, 4)
    z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
    with pytest.raises(ValueError):
        ctx.hdc_quantize(z(4, 100), z(4, 15, d=torch.int32), z(4, 4, d=torch.uint8))
    with pytest.raises(ValueError):
        ctx.hdc_quantize(z(4, 100), z(4, 16, d=torch.int32), z(4, 4, d=torch.uint8), z(5, d=torch.float64))
    with pytest.raises(TypeError):
        ctx.hdc_quantize(z(4, 100).half(), z(4, 16, d=torch.int32), z(4, 4, d=torch.uint8))
    with pytest.raises(TypeError):
        ctx.hdc_dequantize(z(4, 16, d=torch.int32), z(8, 4, d=torch.uint8)[::2], z(4, 100))
    with pytest.raises(ValueError):
        ctx.hdc_search_quantized(z(3, 4, d=torch.int32), z(5, 16, d=torch.int32), z(5, 4, d=torch.uint8), z(5, d=torch.float64), z(3, d=torch.int32))
    with pytest.raises(ValueError):
        ctx.hdc_product_quantized(z(3, 16, d=torch.int32), z(3, 4, d=torch.uint8), z(2, 16, d=torch.int32), z(2, 4, d=torch.uint8), z(2, 3))
    ctx.close()


# ---- together, on another stream, and replayed
def test_train_quantise_search_and_compare_models():
    """The set as a program uses it: training that answers in 4 bits, the rows' way back, inference, rows against rows."""
    rng = np.random.default_rng(11)
    N, C, D = 900, 5, 2000
    cls = words(rng, C, D)
    y = rng.integers(0, C, N).astype(np.int32)
    hv = cls[y] ^ (words(rng, N, D) & words(rng, N, D) | words(rng, N, D) & words(rng, N, D) & words(rng, N, D))
    acc, codes, scales, norm = run_training(hv, y, np.zeros((C, D), np.float32), 100, 2, 1.0)
    ctx = context(D, C)
    dc, ds, dn = dev_u32(codes), torch.from_numpy(scales).cuda(), torch.from_numpy(norm).cuda()
    back, pred = torch.empty((C, D), device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda")
    near = torch.empty((C, C), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h = dev_u32(hv)
    side.wait_stream(torch.cuda.current_stream())
    ctx.hdc_dequantize(dc, ds, back, stream=side)
    ctx.hdc_search_quantized(h, dc, ds, dn, pred, stream=side)
    ctx.hdc_product_quantized(dc, ds, dc, ds, near, stream=side)
    side.synchronize()
    ctx.close()
    v = back.cpu().numpy().astype(np.float64)
    assert np.array_equal(v, oq.values(codes, scales, D))
    assert np.abs(v - acc).max() <= np.abs(acc).max() / 4        # (a step of the largest values is a quarter of them at most)
    assert (pred.cpu().numpy() == y).mean() > 0.99
    got = near.cpu().numpy().astype(np.float64)
    assert np.array_equal(got, got.T)
    assert np.all(np.abs(got - v @ v.T) <= (D + 2) * 2.0 ** -24 * (np.abs(v) @ np.abs(v).T))
    assert np.all(np.abs(np.diag(got) - norm) <= (D + 2) * 2.0 ** -24 * norm)


@pytest.mark.parametrize("N,C,D", [(1, 6, 1000), (70, 5, 2000), (3000, 26, 500), (9, 300, 4100)])
def test_replayed_from_a_graph(N, C, D):
    from paper_2206_04746_amd import binding
    rng = np.random.default_rng(N + D)
    ctx = context(D, C)
    W = (D + 31) // 32
    ctx.hdc_reserve(binding.HDC_RESERVE_ONLINE_BATCHED, max_batch=N)
    x = torch.from_numpy(rows_of("normal", C, D, rng)).cuda()
    hv, y = dev_u32(words(rng, N, D)), torch.from_numpy(rng.integers(0, C, N).astype(np.int32)).cuda()

    def buffers():
        z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
        return dict(codes=z(C, 4 * W, d=torch.int32), scales=z(C, W, d=torch.uint8), norm=z(C, d=torch.float64), back=z(C, D), pred=z(N, d=torch.int32),
                    cos=z(N, C), out=z(C, C), acc=z(C, D), tcodes=z(C, 4 * W, d=torch.int32), tscales=z(C, W, d=torch.uint8), tnorm=z(C, d=torch.float64))

    def step(b):
        ctx.hdc_quantize(x, b["codes"], b["scales"], b["norm"])
        ctx.hdc_dequantize(b["codes"], b["scales"], b["back"])
        ctx.hdc_search_quantized(hv, b["codes"], b["scales"], b["norm"], b["pred"], b["cos"])
        ctx.hdc_product_quantized(b["codes"], b["scales"], b["codes"], b["scales"], b["out"])
        b["acc"].copy_(b["back"])
        ctx.hdc_train_online_quantized(hv, y, b["acc"], b["tcodes"], b["tscales"], b["tnorm"], max(1, N // 2))

    eager, replay = buffers(), buffers()
    step(replay)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step(replay)
    torch.cuda.synchronize()
    for round_ in range(4):
        x.copy_(torch.from_numpy(rows_of("orders" if round_ == 2 else "normal", C, D, rng)).cuda())
        hv.copy_(dev_u32(words(rng, N, D)))
        for v in replay.values():
            v.fill_(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for k in eager:
            assert torch.equal(eager[k], replay[k]), (round_, k)
    ctx.close()
