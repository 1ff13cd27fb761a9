"""Calls with rows of 4-bit floats whose answer must not depend on the way that a call's size takes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import quantized as oq  # noqa: E402

from test_gpu_parity import dev_u32  # noqa: E402
from test_gpu_quantized import U, context, quantized, rows_of, run_training, words  # noqa: E402


def searched(hv, codes, scales, norm, C, D, want_cos):
    """pred and cos (or None) on the host; tables on the device."""
    ctx = context(D, C)
    pred = torch.full((len(hv),), -7, dtype=torch.int32, device="cuda")
    cos = torch.full((len(hv), C), 7.0, dtype=torch.float32, device="cuda") if want_cos else None
    ctx.hdc_search_quantized(dev_u32(hv), codes, scales, norm, pred, cos)
    torch.cuda.synchronize()
    ctx.close()
    return pred.cpu().numpy(), cos.cpu().numpy() if want_cos else None


# ---- cosines that are equal by definition, or differ by one rounding: a row of 0, 1, 2 and 4 times 1.5 is as exact as itself, and its cosine
# the same number but for the roundings of its norm's root, of the product with the sample's and of the quotient.  With whole numbers
# for dot products and norms all that is rounded is what the definition rounds, so classes are equal to the oracle's whatever the call's size.
def rows_of_multiples(C, D, rng, few=5):
    x = rng.choice([0, 1, 2, 4], size=(C, D)) * rng.choice([-1, 1], size=(C, D))
    x[:, ::32] = 4                                                     # (every block has the same scale)
    x = x.astype(np.float64)
    if C > few:
        x[few:] = x[rng.integers(0, few, C - few)]
    x *= rng.choice([1, 1.5], size=(C, 1)) * np.exp2(rng.integers(-3, 4, (C, 1)))
    return x.astype(np.float32)


@pytest.mark.parametrize("want_cos", [False, True])
@pytest.mark.parametrize("N,C,D,far", [
    (70, 10, 400, 0), (70, 30, 400, 0), (70, 40, 400, 0), (9, 300, 1000, 0), (600, 10, 10000, 0), (600, 30, 10000, 0),       # eight waves a row
    (50000, 10, 400, 0), (50000, 30, 400, 0), (50000, 40, 400, 0), (50001, 12, 2048, 0), (50001, 20, 1500, 0),               # fewer waves a row
    (50000, 6, 5000, 0), (50000, 26, 2500, 0), (50000, 40, 2500, 0), (50000, 26, 2500, 12),                                    # ... four of them
    (17000, 100, 400, 0), (25000, 100, 400, 0), (8200, 300, 1021, 0),                                                                          # many classes
    (40, 7, 20600, 0), (40, 20, 14500, 0),                                                                                     # rows in parts
    (70, 10, 400, 12), (70, 40, 400, 12), (50000, 10, 400, 12), (17000, 100, 400, 12), (25000, 100, 400, 12), (40, 7, 20600, 12)])                    # scales far apart
def test_classes_are_those_of_the_definition_whatever_the_size(N, C, D, far, want_cos):
    rng = np.random.default_rng(N + C + D)
    x = rows_of_multiples(C, D, rng)
    if far:                                                            # half of the blocks 2^12 below the others: sums of 44 bits at most
        x[:, np.arange(D) // 32 % 2 == 1] *= 2.0 ** -far
    hv = words(rng, N, D)
    codes, scales, norm = quantized(x)
    v = oq.values(codes.cpu().numpy(), scales.cpu().numpy(), D)
    assert np.array_equal(v, x)                                        # (nothing is rounded)
    assert np.array_equal(norm.cpu().numpy(), (v * v).sum(1))
    pred, _ = searched(hv, codes, scales, norm, C, D, want_cos)
    for n in range(0, N, 4000):
        assert np.array_equal(pred[n:n + 4000], oq.nearest(oq.cosines(hv[n:n + 4000], v, norm.cpu().numpy())))


@pytest.mark.parametrize("N,C,D", [(300, 10, 400), (300, 30, 400), (300, 60, 400)])
def test_training_scores_equal_cosines_as_the_search_does(N, C, D):
    """One batch: the rows that it leaves tell which class was predicted (a wrong one loses about 1 at each of a sample's dimensions)."""
    rng = np.random.default_rng(C)
    x = rows_of_multiples(C, D, rng)
    hv, y = words(rng, N, D), rng.integers(0, C, N).astype(np.int32)
    codes, scales, norm = quantized(x)
    pred, _ = searched(hv, codes, scales, norm, C, D, False)
    got = run_training(hv, y, x, N, 1, 1.0)[0].astype(np.float64)
    cos = oq.cosines(hv, x.astype(np.float64), norm.cpu().numpy())
    weight = np.zeros((N, C))
    at = np.arange(N)
    weight[at, y] = (1.0 - cos[at, y]).astype(np.float32)
    wrong = pred != y
    weight[at[wrong], pred[wrong]] -= (1.0 - cos[at, pred]).astype(np.float32)[wrong]
    want = (x + weight.T @ oq.signs(hv, D)).astype(np.float32)
    # (a weight of at most 2 may be rounded the other way, an element once more)
    assert np.all(np.abs(got - want) <= 2.0 ** -23 * np.abs(want) + 2.0 ** -23 * np.abs(weight).sum(0)[:, None])


# ---- products of more rows than a launch has threads for
def test_product_of_more_rows_than_a_launch_has_threads_for():
    """2^31 + 70 rows of one dimension: 46 GB."""
    N = (1 << 31) + 70
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("no room")
    ctx = context(1)
    codes, scales = torch.zeros((N, 4), dtype=torch.int32, device="cuda"), torch.full((N, 1), 127, dtype=torch.uint8, device="cuda")
    codes[:, 0] = 4                                       # 2
    codes[-100:, 0] = torch.arange(100, device="cuda", dtype=torch.int32) % 8
    codes[:100, 0] = torch.arange(100, device="cuda", dtype=torch.int32) % 8 + 8
    out = torch.full((1, N), -1.0, device="cuda")
    ctx.hdc_product_quantized(codes[:1] * 0 + torch.tensor([[2, 0, 0, 0]], dtype=torch.int32, device="cuda"), scales[:1], codes, scales, out)
    torch.cuda.synchronize()
    ctx.close()
    mags = torch.tensor(oq.MAGNITUDES, dtype=torch.float32, device="cuda")
    at = torch.arange(100, device="cuda") % 8
    assert torch.equal(out[0, :100], -mags[at]) and torch.equal(out[0, -100:], mags[at])
    for n in range(100, N - 100, 1 << 28):
        assert bool((out[0, n:min(n + (1 << 28), N - 100)] == 2.0).all())
    del codes, scales, out
    torch.cuda.empty_cache()

# ---- long rows with so many samples that a block has several tiles of them: rows in parts, and rows that are held by one form of block only
@pytest.mark.parametrize("kind", ["normal", "orders", "none"])
@pytest.mark.parametrize("N,C,D", [(8230, 7, 20481), (8230, 20, 14337), (16420, 40, 14337), (49200, 7, 14400), (49200, 3, 20480), (49200, 5, 20481),
                                   (49153, 12, 14336), (49200, 20, 14400),
                                   (49200, 6, 10240), (49200, 6, 10241)])
def test_long_rows_with_several_tiles_of_samples_a_block(N, C, D, kind):
    """Cosines within their roundings (a sum of W whole numbers, W + 8 roundings of 2^-53, then the one to fp32) and the nearest class, of
    the samples at the ends of the call and some hundreds between."""
    rng = np.random.default_rng(N + C + D)
    x = rows_of("normal" if kind == "none" else kind, C, D, rng)
    if kind == "none":
        x[1, D // 2] = np.nan
    codes, scales, norm = quantized(x)
    hv = words(rng, N, D)
    pred, cos = searched(hv, codes, scales, norm, C, D, True)
    v, norm = oq.values(codes.cpu().numpy(), scales.cpu().numpy(), D), norm.cpu().numpy()
    assert pred.min() >= 0 and pred.max() < C
    some = np.unique(np.concatenate([np.arange(70), np.arange(N - 70, N), rng.integers(0, N, 700)]))
    want = oq.cosines(hv[some], v, norm)
    slack = ((D + 31) // 32 + 8) * U
    got = cos[some].astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.all(np.abs(got - want)[ok] <= 2.0 ** -24 * np.abs(want)[ok] * (1 + 1e-6) + 1.5 * slack)
    order = np.sort(np.where(np.isnan(want), -2, want), axis=1)
    clear = order[:, -1] - order[:, -2] > 3 * slack
    assert np.array_equal(pred[some][clear], oq.nearest(want)[clear])
    # all others: as in calls of so few samples that a block has one tile of them
    own = context(D, C)
    for n in range(0, N, 4096):
        few = torch.empty(min(4096, N - n), dtype=torch.int32, device="cuda")
        of = torch.empty((len(few), C), device="cuda")
        own.hdc_search_quantized(dev_u32(hv[n:n + 4096]), codes, scales, torch.from_numpy(norm).cuda(), few, of)
        assert np.array_equal(few.cpu().numpy(), pred[n:n + 4096])
        # (in as many parts as the form of the block has: the same number but for the last roundings)
        assert np.allclose(of.cpu().numpy(), cos[n:n + 4096], rtol=2.0 ** -23, atol=3 * slack, equal_nan=True)
    own.close()


@pytest.mark.parametrize("N,C,D", [(8230, 7, 20481), (8230, 20, 14337)])
def test_training_on_long_rows_with_several_tiles_of_samples_a_block(N, C, D):
    rng = np.random.default_rng(N + C + D)
    hv, y = words(rng, N, D), rng.integers(0, C, N).astype(np.int32)
    acc = np.rint(30 * rng.normal(size=(C, D))).astype(np.float32)
    got = run_training(hv, y, acc, N, 1, 0.5)[0]
    _, _, v, norm = oq.quantize(acc)
    total, size = np.zeros((C, D)), np.zeros(C)
    for n in range(0, N, 1000):
        h, of = hv[n:n + 1000], y[n:n + 1000]
        cos = oq.cosines(h, v, norm)
        pred, at, weight = oq.nearest(cos), np.arange(len(of)), np.zeros((len(of), C))
        weight[at, of] = (1.0 - cos[at, of]).astype(np.float32)
        wrong = pred != of
        weight[at[wrong], pred[wrong]] = -(0.5 * (1.0 - cos[at, pred])).astype(np.float32)[wrong]
        total += weight.T @ oq.signs(h, D)
        size += np.abs(weight).sum(0)
    want = (acc + total).astype(np.float32)
    assert np.all(np.abs(got.astype(np.float64) - want) <= 2.0 ** -23 * np.abs(want) + 2.0 ** -23 * size[:, None])

# ---- pad bits of samples may be set or not
@pytest.mark.parametrize("kind", ["normal", "orders"])
@pytest.mark.parametrize("N,C,D", [(1, 1, 1), (33, 6, 33), (70, 10, 1001), (70, 26, 4097), (40, 40, 777), (5, 300, 100), (50001, 10, 97), (50001, 26, 500),
                                   (17000, 100, 290), (8200, 300, 1021), (40, 7, 20490), (40, 20, 14345)])
def test_pad_bits_of_samples_count_for_nothing_in_a_search(N, C, D, kind):
    rng = np.random.default_rng(N + C + D)
    codes, scales, norm = quantized(rows_of(kind, C, D, rng))
    hv = words(rng, N, D)
    set_ = hv.copy()
    set_[:, -1] |= rng.integers(0, 1 << 32, N, dtype=np.uint32) << np.uint32(D % 32)
    assert D % 32 and (set_ != hv).any()
    a, b = searched(hv, codes, scales, norm, C, D, True), searched(set_, codes, scales, norm, C, D, True)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("N,C,D,batch", [(50, 3, 33, 20), (300, 26, 333, 300), (300, 40, 1001, 100), (1500, 20, 97, 1500), (20000, 6, 130, 20000), (70, 6, 20490, 40)])
def test_pad_bits_of_samples_count_for_nothing_in_training(N, C, D, batch):
    rng = np.random.default_rng(N + C + D)
    hv, y = words(rng, N, D), rng.integers(0, C, N).astype(np.int32)
    set_ = hv.copy()
    set_[:, -1] |= rng.integers(0, 1 << 32, N, dtype=np.uint32) << np.uint32(D % 32)
    acc = np.rint(10 * rng.normal(size=(C, D))).astype(np.float32)
    for a, b in zip(run_training(hv, y, acc, batch, 1, 0.7), run_training(set_, y, acc, batch, 1, 0.7)):
        assert np.array_equal(a, b)

# ---- products whose partial sums leave fp32: infinite or no number, never a number that is wrong
PRODUCTS = [(10, 30, 600), (300, 200, 600), (30, 40, 300), (600, 600, 513), (1290, 1300, 769), (3000, 3000, 512)]


@pytest.mark.parametrize("M,N,D", PRODUCTS)
@pytest.mark.parametrize("signs", ["equal", "mixed", "halves"])
def test_products_beyond_fp32_are_infinite_or_no_number(M, N, D, signs):
    """Blocks around 2^62 on both sides: sums of magnitudes between far below and far beyond 2^128.  (halves: b's first dimensions are positive,
    the others negative, so that partial sums leave fp32 both ways.)"""
    rng = np.random.default_rng(M + N + D)

    def rows(n, halves=False):
        x = rng.normal(size=(n, D)) if signs == "mixed" else np.abs(rng.normal(size=(n, D)))
        x[:, D // 2:] *= -1 if halves else 1
        return (x * np.exp2(rng.integers(54, 64, (n, 1)))).astype(np.float32)
    ctx = context(D)
    a, sa, _ = quantized(rows(M), ctx, norm=False)
    b, sb, _ = quantized(rows(N, signs == "halves"), ctx, norm=False)
    out = torch.full((M, N), 3.0, device="cuda")
    ctx.hdc_product_quantized(a, sa, b, sb, out)
    torch.cuda.synchronize()
    ctx.close()
    va, vb = oq.values(a.cpu().numpy(), sa.cpu().numpy(), D), oq.values(b.cpu().numpy(), sb.cpu().numpy(), D)
    got, want, size = out.cpu().numpy().astype(np.float64), va @ vb.T, np.abs(va) @ np.abs(vb).T
    slack = (D + 2) * 2.0 ** -24 * size
    number = np.isfinite(got)
    assert np.all(np.abs(got - want)[number] <= slack[number])                  # what is a number is right
    fits = size * (1 + (D + 2) * 2.0 ** -24) < 2.0 ** 128 - 2.0 ** 103
    assert np.all(number[fits]) and fits.any() and (~fits).any()                # and where no partial sum can leave fp32 it is one
    beyond = ~number & ~np.isnan(got)
    assert np.all(size[beyond] >= 2.0 ** 127)
    if signs == "equal":
        assert not np.isnan(got).any() and np.all(got[want - slack > 2.0 ** 128] == np.inf)


@pytest.mark.parametrize("M,N,D", PRODUCTS)
@pytest.mark.parametrize("run", [32, 1])
def test_zeros_beside_huge_values_add_nothing(M, N, D, run):
    """Of every two runs of dimensions (blocks, or single ones) a has huge values in the first and b in the second; the last block has products of 1
    on every dimension."""
    W = (D + 31) // 32
    x, y = np.zeros((M, D), np.float32), np.zeros((N, D), np.float32)
    block = np.arange(D) // 32
    x[:, np.arange(D) // run % 2 == 0], y[:, np.arange(D) // run % 2 == 1] = 3.0e38, -3.0e38
    x[:, block == W - 1] = y[:, block == W - 1] = 1.0
    ctx = context(D)
    a, sa, _ = quantized(x, ctx, norm=False)
    b, sb, _ = quantized(y, ctx, norm=False)
    out = torch.full((M, N), 3.0, device="cuda")
    ctx.hdc_product_quantized(a, sa, b, sb, out)
    torch.cuda.synchronize()
    ctx.close()
    assert bool((out == float((block == W - 1).sum())).all())
