"""The kernel for the rows that pass through the caches keeps its registers and its arguments where they are: what it calls for rows of too many
equal values saves registers of its own, but nothing in the kernel touches memory for it.  Reads the listing of the library built
here; needs no GPU."""
from test_kernel_code import _named, kernels      # noqa: F401  (the fixture)


def test_wide_rows_keep_their_registers(kernels):  # noqa: F811
    for name, code in _named(kernels, "sample_bf16_wide_kernel").items():
        assert not [c for c in code if c.startswith("scratch_")], name
