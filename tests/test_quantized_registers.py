"""Registers and scratch of the kernels of 4-bit class rows, as their launch bounds and comments have them."""
import re

from test_kernel_registers import kernels, of  # noqa: F401  (the fixture)


def test_searches_hold_their_rows_in_registers(kernels):  # noqa: F811
    some = of(kernels, "search_quantized_kernel")
    modes = [re.search(r"ILi(\d+)ELi(\d+)ELi(\d)ELb(\d)ELi(\d)E", n).groups() for n in some]
    assert not any(c == "16" and mode == "1" for c, _, _, _, mode in modes)      # dot products: of more than 32 classes only
    for (name, f), (_, steps, _, _, mode) in zip(some.items(), modes):          # two waves a SIMD
        assert f["vgpr_count"] <= 256 and f["agpr_count"] == 0, (name, f)
        # (28 steps, rows of 12289 to 14336 dimensions: 4 registers of a search, 10 of a training batch)
        assert f["vgpr_spill_count"] <= ({"0": 4, "2": 10}.get(mode, 0) if steps == "28" else 0), (name, f)


def test_search_of_many_classes_spills_after_its_loop_only_so_much(kernels):  # noqa: F811
    for name, f in of(kernels, "search_many_kernel").items():
        assert f["vgpr_count"] <= 256 and f["private_segment_fixed_size"] <= 216, (name, f)


def test_products_and_quantisation_do_not_spill(kernels):  # noqa: F811
    for name, f in of(kernels, "product_(few|tiles)_kernel|quantize_rows_kernel|scan_kernel|nearest_kernel").items():
        assert f["private_segment_fixed_size"] == 0 and f["vgpr_spill_count"] == 0, (name, f)
    for name, f in of(kernels, "product_tiles_kernelILi4ELi4ELi1E").items():      # sixteen tiles of sums a wave
        assert f["agpr_count"] == 256, (name, f)
