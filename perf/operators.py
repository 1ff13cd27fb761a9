"""Class rows in 4-bit floats with a scale for every 32 dimensions, as cases to be timed: quantisation and its way back,
inference and products on such rows, training of rows that are answered with in this form.

A row of D dimensions has W = ceil(D / 32) blocks; block w is dimensions 32 w to 32 w + 31, which are word w of a
hypervector.  A block has a scale byte s, worth 2^(s - 127) (255: no number), and four 32-bit words of codes: nibble j of
word r is dimension 32 w + 4 j + r, its top bit the sign, the others one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.

Operations
  quantize   rows of 32-bit floats to codes, scales and squared norms, and back to the values that these stand for
  search     cosines of hypervectors with such class rows, and the nearest class
  product    scalar products of such rows with one another
  train      online training in batches, the rows quantised anew before each, the updates taken by the 32-bit rows
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"


def _case(op, D, N, C=0, cos=True, epochs=1, batch=0):
    return dict(op=op, D=D, N=N, C=C, cos=cos, epochs=epochs, batch=batch)


def listed():
    return [
        # the class rows of the activity model after training, looked at in 4 bits: launches and latency
        dict(_case("quantize", D=10000, N=6), name="quantize-ucihar"),
        # a training set's worth of real-valued rows (sums of a few hypervectors), an odd length
        dict(_case("quantize", D=9999, N=6238), name="quantize-many"),
        # one window at a time, as a wearable or a request handler classifies it
        dict(_case("search", D=10000, N=1, C=6), name="search-one"),
        # the test set of the activity model, cosines kept for a confidence
        dict(_case("search", D=10000, N=2947, C=6), name="search-ucihar"),
        # a long stream of encoded rows against the spoken-letter model
        dict(_case("search", D=10000, N=200000, C=26), name="search-stream"),
        # as many classes as a model may have (a retrieval of prototypes), an odd number of queries and dimensions
        dict(_case("search", D=8191, N=16001, C=1024), name="search-prototypes"),
        # one real-valued query (the sum of a window of hypervectors) with the class rows
        dict(_case("product", D=10000, N=1, C=26), name="product-one"),
        # a test set of them
        dict(_case("product", D=10000, N=1559, C=26), name="product-isolet"),
        # rows with rows, many of both: how near prototypes of one model come to those of another; the largest
        dict(_case("product", D=9999, N=8191, C=4093), name="product-many"),
        # the tiny model, retrained from its class sums in small batches: where the dependent steps count
        dict(_case("train", D=1024, N=2000, C=5, batch=32), name="train-tiny"),
        # the activity model, three passes, rows updated after every 64 windows
        dict(_case("train", D=10000, N=7352, C=6, epochs=3, batch=64), name="train-ucihar"),
        # the spoken-letter model in large batches
        dict(_case("train", D=10000, N=6238, C=26, batch=1024), name="train-isolet"),
    ]


def _log(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "search", "search", "product", "product", "train"])
    D = _log(rng, 500, 16384)
    if op == "quantize":
        return _case(op, D=D, N=_log(rng, 1, min(60000, 62000000 // D)))
    if op == "search":
        C = _log(rng, 2, 1024)
        return _case(op, D=D, C=C, N=_log(rng, 1, min(200000, int(2e9 / D), int(1.3e11 / (C * D)))), cos=rng.random() < 0.75)
    if op == "product":
        C = _log(rng, 1, 4096)
        return _case(op, D=D, C=C, N=_log(rng, 1, min(16384, int(3.2e11 / (C * D)))))
    D = _log(rng, 500, 12000)
    N = _log(rng, 300, 8000)
    return _case(op, D=D, C=_log(rng, 2, 32), N=N, epochs=rng.choice([1, 1, 2]), batch=_log(rng, 32, min(N, 4096)))


def work(case):
    """Inputs read once, outputs written once; a row of W blocks has 17 W bytes."""
    D, N, C, e = case["D"], case["N"], case["C"], case["epochs"]
    W = (D + 31) // 32
    if case["op"] == "quantize":      # rows in; codes, scales, norms and the values out
        return {"bytes": 8 * N * D + 17 * N * W + 8 * N, "flops": 4 * N * D}
    if case["op"] == "search":
        return {"bytes": 4 * N * W + 17 * C * W + 8 * C + 4 * N * (1 + C * case["cos"]), "flops": 2 * N * C * D}
    if case["op"] == "product":
        return {"bytes": 17 * W * (N + C) + 4 * N * C, "flops": 2 * N * C * D}
    # every pass reads the samples; scores of every class, an update of a sample's own class at least
    return {"bytes": e * N * (4 * W + 4) + 12 * C * D + 17 * C * W, "flops": e * N * (2 * C * D + 2 * D)}


# ------------------------------------------------------------------------------------- plain forms
def _quantise(x):
    """Scale bytes [N][W] and codes [N][W][32], in the order of the dimensions, of rows [N][D]."""
    N, D = x.shape
    W = (D + 31) // 32
    x = torch.nn.functional.pad(x, (0, 32 * W - D)).view(N, W, 32)
    most = x.abs().amax(2).double()
    ex = torch.where(most > 0, torch.frexp(most).exponent - 3, -127).clamp(min=-127)   # floor(log2) less 2
    fine = torch.isfinite(most)
    v = x.abs().double() * ((1023 - ex.long()) << 52).view(torch.float64)[:, :, None]  # relative to the scale
    code = (v > 0.25).to(torch.uint8)                                                  # nearest, ties to even codes
    for up in (v >= 0.75, v > 1.25, v >= 1.75, v > 2.5, v >= 3.5, v > 5.0):
        code += up
    code = (code + 8 * torch.signbit(x)) * fine[:, :, None]
    return torch.where(fine, ex + 127, 255).to(torch.uint8), code.to(torch.uint8)


def _values(scales, code, D):
    """The values, 64 bits, that scales and codes stand for: [N][D]."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=scales.device)
    unit = ((scales.long() + 896) << 52).view(torch.float64)
    unit = torch.where(scales == 255, math.nan, unit)
    return (grid[code.long()] * unit[:, :, None]).reshape(code.shape[0], -1)[:, :D]


def _packed(code):
    """Codes [N][W][32] as words [N][4 W]: nibble j of word r is dimension 4 j + r."""
    N, W = code.shape[:2]
    shift = 4 * torch.arange(8, device=code.device)
    words = (code.view(N, W, 8, 4).long() << shift[:, None]).sum(2)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).reshape(N, 4 * W)


def _unpacked(words):
    """Codes [N][W][32] of words [N][4 W]."""
    N, W = words.shape[0], words.shape[1] // 4
    shift = 4 * torch.arange(8, device=words.device, dtype=torch.int32)
    return ((words.view(N, W, 1, 4) >> shift[:, None]) & 15).to(torch.uint8).reshape(N, W, 32)


def _signs(hv, D):
    """Bits as +-1 in 64 bits: [n][D]."""
    bits = (hv[:, :, None] >> torch.arange(32, device=hv.device, dtype=torch.int32)) & 1
    return bits.reshape(hv.shape[0], -1)[:, :D].double().mul_(2).sub_(1)


def _cosines(dot, norm, D):
    """Cosines of the scalar products; a row of zeros has 0."""
    return torch.where(norm == 0, 0.0, dot / (norm.sqrt() * math.sqrt(D)))


def _nearest(cos):
    """The lowest class of the largest cosine; one that is no number is below all others."""
    return torch.where(torch.isnan(cos), -math.inf, cos).argmax(1).to(torch.int32)


# ------------------------------------------------------------------------------------- inputs
def _words(g, n, W):
    return torch.randint(-(1 << 31), 1 << 31, (n, W), device=DEV, generator=g, dtype=torch.int32)


def _samples(case, g):
    """Encoded rows of a task: classes that share a common part, samples a quarter of whose bits differ from their class."""
    D, N, C = case["D"], case["N"], case["C"]
    W = (D + 31) // 32
    cls = (_words(g, C, W) & _words(g, C, W)) ^ _words(g, 1, W)
    y = torch.randint(0, C, (N,), device=DEV, generator=g, dtype=torch.int32)
    hv = _words(g, N, W).bitwise_and_(_words(g, N, W)).bitwise_xor_(cls[y.long()])
    if D % 32:
        hv[:, -1] &= (1 << (D % 32)) - 1
        cls[:, -1] &= (1 << (D % 32)) - 1
    return hv, y, cls


def _context(case):
    """A model of one feature carries D and C."""
    from paper_2206_04746_amd import binding

    W = (case["D"] + 31) // 32
    zero = lambda n: np.zeros((n, W), np.uint32)  # noqa: E731
    return binding.Context(case["D"], 1, 2, max(1, min(case["C"], 1024)), zero(1), zero(2), zero(1)[0], None, None, "u8")


def prepare(case, seed):
    op, D, N, C = case["op"], case["D"], case["N"], case["C"]
    W = (D + 31) // 32
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=DEV)  # noqa: E731
    randn = lambda *shape: torch.randn(shape, device=DEV, generator=g)  # noqa: E731
    s = dict(case=case, ctx=_context(case) if own else None)
    if op == "quantize":   # sums of weighted hypervectors, of a size that differs from row to row
        s["rows"] = randn(N, D).mul_(12.0 * torch.exp(randn(N, 1)))
        s.update(codes=new(N, 4 * W, dtype=torch.int32), scales=new(N, W, dtype=torch.uint8), norm=new(N, dtype=torch.float64), back=new(N, D))
    elif op == "search":   # rows as training leaves them: the class's bits under the sums of other samples' noise
        s["hv"], _, cls = _samples(case, g)
        scales, code = _quantise((20.0 * _signs(cls, D)).float() + 12.0 * randn(C, D))
        s.update(codes=_packed(code), scales=scales, norm=_values(scales, code, D).square().sum(1))
        s.update(pred=new(N, dtype=torch.int32), cos=new(N, C) if case["cos"] else None)
    elif op == "product":   # rows of two sets with something in common
        common = randn(1, D)
        for name, n in (("a", N), ("b", C)):
            scales, code = _quantise(randn(n, D).add_(common).mul_(12.0 * torch.exp(randn(n, 1))))
            s.update({name + "_codes": _packed(code), name + "_scales": scales})
        s["out"] = new(N, C)
    else:   # class sums of the samples, whose labels are wrong now and then
        s["hv"], y, _ = _samples(case, g)
        wrong = torch.rand(N, device=DEV, generator=g) < 0.1
        s["y"] = torch.where(wrong, torch.randint(0, C, (N,), device=DEV, generator=g, dtype=torch.int32), y)
        s["sums"] = new(C, D)
        for n in range(0, N, 4096):
            part = _signs(s["hv"][n:n + 4096], D)
            s["sums"] += (torch.eye(C, device=DEV, dtype=torch.float64)[:, s["y"][n:n + 4096].long()] @ part).float()
        s.update(acc=new(C, D), codes=new(C, 4 * W, dtype=torch.int32), scales=new(C, W, dtype=torch.uint8), norm=new(C, dtype=torch.float64), back=new(C, D))
        if own:
            s["ctx"].hdc_reserve(2, max_batch=case["batch"])   # HDC_RESERVE_ONLINE_BATCHED
    return s


# ------------------------------------------------------------------------------------- a pass
def run(s):
    case = s["case"]
    op, D = case["op"], case["D"]
    if own:
        ctx = s["ctx"]
        if op == "quantize":
            ctx.hdc_quantize(s["rows"], s["codes"], s["scales"], s["norm"])
            ctx.hdc_dequantize(s["codes"], s["scales"], s["back"])
            return s["back"], s["norm"]
        if op == "search":
            ctx.hdc_search_quantized(s["hv"], s["codes"], s["scales"], s["norm"], s["pred"], s["cos"])
            return (s["pred"], s["cos"]) if case["cos"] else s["pred"]
        if op == "product":
            ctx.hdc_product_quantized(s["a_codes"], s["a_scales"], s["b_codes"], s["b_scales"], s["out"])
            return s["out"]
        s["acc"].copy_(s["sums"])
        ctx.hdc_train_online_quantized(s["hv"], s["y"], s["acc"], s["codes"], s["scales"], s["norm"], case["batch"], case["epochs"], 1.0)
        ctx.hdc_dequantize(s["codes"], s["scales"], s["back"])
        return s["acc"], s["back"], s["norm"]
    if op == "quantize":
        values = _values(*_quantise(s["rows"]), D)
        return values.float(), values.square().sum(1)
    if op == "search":
        # in 64 bits: nearest classes of near cosines have to be told apart; 4096 samples' signs at a time
        rows = _values(s["scales"], _unpacked(s["codes"]), D).t().contiguous()
        dot = torch.cat([_signs(hv, D) @ rows for hv in s["hv"].split(4096)])
        cos = _cosines(dot, s["norm"], D)
        return (_nearest(cos), cos.float()) if case["cos"] else _nearest(cos)
    if op == "product":
        a = _values(s["a_scales"], _unpacked(s["a_codes"]), D).float()
        b = _values(s["b_scales"], _unpacked(s["b_codes"]), D).float()
        return a @ b.t().contiguous()
    acc, C = s["sums"].clone(), case["C"]
    classes = torch.arange(C, device=DEV)
    for _ in range(case["epochs"]):
        for hv, y in zip(s["hv"].split(case["batch"]), s["y"].split(case["batch"])):
            signs, values = _signs(hv, D), _values(*_quantise(acc), D)
            cos = _cosines(signs @ values.t().contiguous(), values.square().sum(1), D)
            pred = _nearest(cos)
            of = lambda c: cos.gather(1, c.long()[:, None])  # noqa: E731
            plus = (classes == y[:, None]) * (1 - of(y)).float().double()       # weights are 32-bit floats
            minus = ((classes == pred[:, None]) & (pred != y)[:, None]) * (1 - of(pred)).float().double()
            acc = (acc.double() + (plus - minus).t().contiguous() @ signs).float()
    values = _values(*_quantise(acc), D)
    return acc, values.float(), values.square().sum(1)


# ------------------------------------------------------------------------------------- in 64 bits, from the definition
_GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def _numpy_rows(x):
    """The values, 64 bits, to which rows are quantised: by the steps between the values of each range."""
    N, D = x.shape
    W = (D + 31) // 32
    out = np.zeros((N, W * 32))
    out[:, :D] = x
    out = out.reshape(N, W, 32)
    most = np.abs(out).max(2)
    unit = np.exp2(np.maximum(np.floor(np.log2(np.maximum(most, 2.0 ** -140))), -125) - 2)   # (log2 of a float just below a power of two)
    unit = np.where(most < 4 * unit, np.maximum(unit / 2, 2.0 ** -127), unit)
    v = np.abs(out) / unit[:, :, None]
    step = np.where(v < 2, 0.5, np.where(v < 4, 1.0, 2.0))
    v = np.minimum(np.rint(v / step) * step, 6.0) * unit[:, :, None]
    return (np.copysign(v, out)).reshape(N, -1)[:, :D]


def _numpy_values(codes, scales, D):
    N, W = scales.shape
    nibbles = codes.view(np.uint8).reshape(N, W, 4, 4, 1) >> np.array([0, 4], np.uint8) & 15     # [N][W][word][byte][half]
    nibbles = nibbles.reshape(N, W, 4, 8).transpose(0, 1, 3, 2).reshape(N, W, 32)
    v = _GRID[nibbles & 7] * np.where(nibbles & 8, -1.0, 1.0) * np.exp2(scales.astype(np.float64) - 127)[:, :, None]
    return v.reshape(N, -1)[:, :D]


def _numpy_bits(hv, D):
    return np.unpackbits(hv.view(np.uint8), axis=1, bitorder="little")[:, :D]


def exact(case, seed):
    op, D, N, C = case["op"], case["D"], case["N"], case["C"]
    s = prepare(case, seed)
    host = lambda k: s[k].cpu().numpy()  # noqa: E731
    if op == "quantize":
        v = np.concatenate([_numpy_rows(r) for r in np.array_split(host("rows"), max(1, N // 256))])
        return v, np.square(v).sum(1)
    if op == "search":
        if N * D > 4e8 or N * C * D > 2e11:
            return None     # (host time)
        v = _numpy_values(host("codes"), host("scales"), D)
        norm, total = np.square(v).sum(1), v.sum(1)
        # a set bit counts for the value, one that is not set against it
        cos = np.concatenate([(2 * (_numpy_bits(hv, D).astype(np.float64) @ v.T) - total) / np.sqrt(norm * D)
                              for hv in np.array_split(host("hv"), max(1, N // 1024))])
        pred = cos.argmax(1).astype(np.int32)
        return (pred, cos) if case["cos"] else pred
    if op == "product":
        if N * C * D > 4e11:
            return None     # (host time)
        return _numpy_values(host("a_codes"), host("a_scales"), D) @ _numpy_values(host("b_codes"), host("b_scales"), D).T
    acc, hv, y = host("sums"), host("hv"), host("y")
    if case["epochs"] * -(-N // case["batch"]) * C * D > 3e8 or N * D * C * case["epochs"] > 1e10:
        return None         # (host time)
    for _ in range(case["epochs"]):
        for n in range(0, N, case["batch"]):
            bits, label = _numpy_bits(hv[n:n + case["batch"]], D) * 2.0 - 1.0, y[n:n + case["batch"]]
            v = _numpy_rows(acc)
            size = np.sqrt(np.square(v).sum(1))
            cos = bits @ v.T / np.where(size > 0, size, 1.0) / np.sqrt(D)
            pred, at = cos.argmax(1), np.arange(len(label))
            weight = np.zeros((len(label), C))
            weight[at, label] = (1 - cos[at, label]).astype(np.float32)
            miss = pred != label
            weight[at[miss], pred[miss]] -= (1 - cos[at, pred]).astype(np.float32)[miss]
            acc = (acc + weight.T @ bits).astype(np.float32)
    v = _numpy_rows(acc)
    return acc, v, np.square(v).sum(1)
