"""What the kernels of trees and sampling must not contain: registers spilled to memory in the loops, and (trees) loads through flat
pointers, each of which is waited for together with everything in flight.  Reads the listing of the library built here; needs no GPU."""
from test_kernel_code import _named, kernels      # noqa: F401  (the fixture)


def test_tree_decode_keeps_its_registers(kernels):  # noqa: F811
    for name, code in _named(kernels, "tree_kernel").items():
        assert not [c for c in code if c.startswith(("scratch_", "flat_"))], name


def test_tree_decode_stages_by_dma(kernels):  # noqa: F811
    for name, code in _named(kernels, "tree_kernel").items():
        assert [c for c in code if c.startswith("global_load_lds_dwordx4")], name


def test_sampling_keeps_its_registers(kernels):  # noqa: F811
    for part in ("sample_f32_kernel", "sample_bf16_kernel", "sample_bf16_long_kernel"):
        for name, code in _named(kernels, part).items():
            assert not [c for c in code if c.startswith("scratch_")], name
