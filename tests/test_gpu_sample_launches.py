"""sp_sample on both sides of every vocabulary at which the launch takes another kernel, and up to the largest vocabulary."""
import gc

import numpy as np
import pytest

import sp_synth
from paper_2404_06910_amd import binding as B

from test_gpu_sample import _check, _params, _sample

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


# bf16: rows in registers up to 32768 and 57344 tokens, counted up to 131072, then searched; fp32: one kernel
@pytest.mark.parametrize("dtype,vocab", [("bf16", v) for v in (32768, 32769, 57344, 57345, 65535, 65536, 131071, 131072, 131073, 152064, 256000)]
                         + [("f32", v) for v in (131073, 256000)])
@pytest.mark.parametrize("what", ["random", "equal", "masked"])
def test_both_sides_of_a_launch(ctx, dtype, vocab, what):
    rng = np.random.default_rng(vocab)
    rows = 10
    x = rng.standard_normal((rows, vocab), dtype=np.float32) * np.float32(3)
    if what == "equal":                                     # more of one value than a 16-bit count holds, from 65536 tokens on
        x[:] = -2.25
        x[::2, vocab // 3] = 1.0
    elif what == "masked":
        x[:, rng.random(vocab) < 0.95] = -np.inf
        x[:, -1] = 6.0
    x = sp_synth.round_to_dtype(x, dtype)
    u = rng.random(rows).astype(np.float32)
    sets = _params(rng, rows)
    print("case:", dtype, vocab, what, flush=True)
    # of equal weights every border is a multiple, and half of the draws of a cut may lie on one
    _check(x, u, _sample(ctx, x, u, dtype, **sets), least_sure=0.5 if what == "equal" else 0.8, **sets)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [(1 << 20) + 1, 1 << 24])
def test_the_largest_vocabularies(ctx, dtype, vocab):
    """tens of tokens have all the weight: a border between two of them is further away than the weights' resolution, 2^-38 at 2^24 tokens"""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, vocab), dtype=np.float32) - 40
    at = rng.choice(vocab, (4, 60))
    at[:, 0] = vocab - 1
    np.put_along_axis(x, at, np.float32(4) + 2 * rng.standard_normal((4, 60), dtype=np.float32), 1)
    x = sp_synth.round_to_dtype(x, dtype)
    u = np.array([0.15, 0.5, 0.8, 0.97], np.float32)
    f = lambda *a: np.array(a, np.float32)
    sets = dict(temperature=f(1, 0.7, 0, 1.3), top_k=np.array([0, 40, 0, 0], np.int32), top_p=f(1, 0.9, 1, 0.8), min_p=f(0, 0, 0, 0.01))
    if vocab > 1 << 21:                                 # a row takes seconds on the host
        x, u, sets = x[:2], u[:2], {n: a[:2] for n, a in sets.items()}
    print("case:", dtype, vocab, flush=True)
    _check(x, u, _sample(ctx, x, u, dtype, **sets), least_sure=0.75, **sets)
