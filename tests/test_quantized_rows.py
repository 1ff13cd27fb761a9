"""Rows of 4-bit floats without a GPU: the oracle's quantisation on values worked out by hand, and every call that the entry
points refuse (they look at their arguments before they touch the context or the device)."""
import ctypes

import numpy as np
import pytest

from oracle import quantized as oq


def test_oracle_on_a_block_worked_out_by_hand():
    # the largest magnitude is 7: floor(log2) is 2, the scale 2^0; 7 is beyond 6
    x = np.zeros((1, 33), np.float32)
    x[0, :12] = [7, -7, 0.25, 0.2500001, 0.75, -1.25, 1.75, 2.5, 3.5, 5, -5.0000005, -0.1]
    x[0, 32] = -3 * 2.0 ** 20
    codes, scales, v, norm = oq.quantize(x)
    assert list(v[0, :12]) == [6, -6, 0, 0.5, 1, -1, 2, 2, 4, 4, -6, 0]
    assert list(scales[0]) == [127, 127 + 21 - 2] and v[0, 32] == -3 * 2.0 ** 20
    assert norm[0] == 36 + 36 + 0.25 + 1 + 1 + 4 + 4 + 16 + 16 + 36 + 9 * 2.0 ** 40
    # dimensions 0, 4, 8 are nibbles 0, 1, 2 of word 0; dimension 1, 5, 9 of word 1, and so on
    assert list(codes[0, :4]) == [0x627, 0x6AF, 0xF40, 0x841]
    assert list(codes[0, 4:]) == [0xF, 0, 0, 0]     # -6 x 2^19
    assert np.signbit(v[0, 11])


@pytest.mark.parametrize("value,scale,is_", [(0.0, 0, 0.0), (2.0 ** -149, 0, 0.0), (2.0 ** -128, 0, 2.0 ** -128), (2.0 ** -126, 0, 2.0 ** -126),
                                             (2.0 ** -124, 1, 2.0 ** -124), (3.4028235e38, 252, 1.5 * 2.0 ** 127), (np.inf, 255, np.nan), (np.nan, 255, np.nan)])
def test_oracle_at_the_ends_of_the_range(value, scale, is_):
    _, scales, v, norm = oq.quantize(np.full((1, 5), value, np.float32))
    assert scales[0, 0] == scale
    assert np.array_equal(v, np.full((1, 5), is_), equal_nan=True)


@pytest.fixture(scope="module")
def calls():
    """name -> (function, valid arguments): pointers that are never followed, a context that is never looked into."""
    from paper_2206_04746_amd import binding
    lib, ctx, p = binding.lib, ctypes.create_string_buffer(1 << 16), ctypes.c_void_p(4096)
    c = ctypes.cast(ctx, ctypes.c_void_p)
    rows = dict(ctx=c, rows=p, N=1, codes=p, scales=p, norm=p, stream=None)
    return ctx, {
        "hdc_quantize": (lib.hdc_quantize, rows),
        "hdc_dequantize": (lib.hdc_dequantize, dict(ctx=c, codes=p, scales=p, N=1, rows=p, stream=None)),
        "hdc_search_quantized": (lib.hdc_search_quantized, dict(ctx=c, hv=p, N=1, codes=p, scales=p, norm=p, cos=p, pred=p, stream=None)),
        "hdc_product_quantized": (lib.hdc_product_quantized, dict(ctx=c, a=p, sa=p, M=1, b=p, sb=p, N=1, out=p, stream=None)),
        "hdc_train_online_quantized": (lib.hdc_train_online_quantized, dict(ctx=c, hv=p, labels=p, N=1, epochs=1, lr=1.0, batch=1, acc=p, codes=p,
                                                                            scales=p, norm=p, stream=None)),
    }


REFUSED = {
    "hdc_quantize": [("ctx", None), ("rows", None), ("codes", None), ("scales", None), ("N", -1), ("rows", 4098), ("codes", 4104), ("norm", 4100)],
    "hdc_dequantize": [("ctx", None), ("rows", None), ("codes", None), ("scales", None), ("N", -1), ("rows", 4098), ("codes", 4100)],
    "hdc_search_quantized": [("ctx", None), ("hv", None), ("codes", None), ("scales", None), ("norm", None), ("pred", None), ("N", -5), ("hv", 4097),
                             ("codes", 4104), ("norm", 4100), ("cos", 4098), ("pred", 4099)],
    "hdc_product_quantized": [("ctx", None), ("a", None), ("sa", None), ("b", None), ("sb", None), ("out", None), ("M", -1), ("N", -1), ("a", 4104),
                              ("b", 4100), ("out", 4098)],
    "hdc_train_online_quantized": [("ctx", None), ("hv", None), ("labels", None), ("acc", None), ("codes", None), ("scales", None), ("N", -1),
                                   ("epochs", -1), ("batch", 0), ("hv", 4098), ("labels", 4098), ("acc", 4098), ("codes", 4104), ("norm", 4100)],
}


@pytest.mark.parametrize("name,field,value", [(n, f, v) for n, some in REFUSED.items() for f, v in some])
def test_refusals(calls, name, field, value):
    from paper_2206_04746_amd import binding
    fn, args = calls[1][name]
    given = dict(args)
    given[field] = ctypes.c_void_p(value) if isinstance(value, int) and value > 1 else value
    assert fn(*given.values()) == binding.HDC_EINVAL


@pytest.mark.parametrize("name,field", [("hdc_quantize", "N"), ("hdc_dequantize", "N"), ("hdc_search_quantized", "N"), ("hdc_product_quantized", "M"),
                                        ("hdc_product_quantized", "N"), ("hdc_train_online_quantized", "N"), ("hdc_train_online_quantized", "epochs")])
def test_nothing_to_do_is_a_success_whatever_the_pointers(calls, name, field):
    from paper_2206_04746_amd import binding
    fn, args = calls[1][name]
    given = {k: None if isinstance(v, ctypes.c_void_p) and k != "ctx" else v for k, v in args.items()}
    given[field] = 0
    assert fn(*given.values()) == binding.HDC_OK
