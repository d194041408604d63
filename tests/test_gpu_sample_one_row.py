"""sp_sample of one row: it has no next one, so its stride may be anything, and nothing behind it is read into the result."""
import gc

import numpy as np
import pytest
import torch

import sp_synth
from oracle import sp_oracle_tree as ort
from paper_2404_06910_amd import binding as B

from gpu_util import TORCH_DT, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 7, 9, 1001, 50257, 70001])
def test_a_row_of_any_stride(ctx, dtype, vocab):
    x = sp_synth.round_to_dtype(np.random.default_rng(vocab).standard_normal((1, vocab), dtype=np.float32), dtype)
    flat = torch.full((vocab + 8,), float("inf"), dtype=TORCH_DT[dtype], device="cuda")
    flat[:vocab] = dev(x, dtype)[0]
    token, logprob = torch.full((1,), -7, dtype=torch.int32, device="cuda"), torch.full((1,), 7.0, device="cuda")
    for u in (0.1, 0.55, 0.9):
        want, lp, margin = ort.sample_row(x[0], np.float32(u))
        assert margin > 2.0 ** -45
        for stride in (vocab, vocab + 1, 0, 3):
            ctx.sp_sample(torch.as_strided(flat, (1, vocab), (stride, 1)), dev(np.array([u], np.float32)), token, logprob)
            torch.cuda.synchronize()
            # the quotient's logarithm in 64 bits, then one rounding to 32
            assert int(token) == want and abs(float(logprob) - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -45
