"""sp_tree_decode in bf16: the softmax weights keep their bits through the second product.  A result is off by its own rounding, half a
step of bf16, and by what the weights and their sums are off, which is less than a hundredth of that."""
import gc

import numpy as np
import pytest
import torch

from oracle import sp_oracle_tree as ort
from paper_2404_06910_amd import binding as B

from gpu_util import dev
from tree_util import TreeCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


# one or two tiles of rows to a wave, waves for rows and for keys, lists that are cut and that are not
@pytest.mark.parametrize("heads,N", [((4, 4, 64), 1), ((4, 4, 128), 12), ((8, 2, 128), 7), ((8, 2, 64), 12), ((16, 2, 128), 33),
                                     ((20, 1, 64), 64)])
@pytest.mark.parametrize("prompts", [2, 40])
@pytest.mark.parametrize("bias", [False, True], ids=["", "bias"])
def test_results_are_rounded_once(ctx, heads, N, prompts, bias):
    c = TreeCase("bf16", *heads, N, B=prompts, preamble=150, resp=(20, 60), bias=bias, seed=N, n_nodes=[N] * prompts)
    print("case:", heads, N, prompts, bias, flush=True)
    t = c.upload()
    c.call(ctx, c.plan(ctx), t)
    torch.cuda.synchronize()
    got = t["o"].float().cpu().numpy()
    eps = 2.0 ** -24
    for b in (0, prompts - 1):
        K, V, pos = c.old_keys(b)
        o, absum, big = ort.tree_attention(c.q[b], c.kn[b], c.vn[b], K, V, c.parent[b], c.scale, c.slopes,
                                           None if c.new_pos is None else c.new_pos[b], pos)
        # Scores and sums as in TreeCase.check, the sums over two products a key; a weight is off by 2^-15 (its upper half leaves
        # less than 2^-7 + 2^-10 of it, which is rounded to eight bits); then the one rounding.
        off = absum * (2.0 ** -15 + eps * (2 * (heads[2] + 8) * 1.45 * big[..., None] + 2 * (len(K) + N) + 16))
        tol = off + 2.0 ** -8 * (np.abs(o) + off)
        assert (np.abs(got[b] - o) <= tol).all(), "prompt %d: %.3g of the bound" % (b, (np.abs(got[b] - o) / tol).max())


@pytest.mark.parametrize("heads,N", [((4, 4, 64), 3), ((8, 2, 128), 12), ((20, 1, 64), 30)])
def test_an_infinite_value_in_the_cache(ctx, heads, N):
    """every node sees the cached key, so that all have its infinity, and none NaN; -inf and a NaN in other dims likewise"""
    c = TreeCase("bf16", *heads, N, preamble=300, resp=(40, 90), seed=4, n_nodes=[N, N - 1])
    c.q *= 0.25                                             # no weight falls below what a float holds
    t = c.upload()
    x = torch.full((heads[1],), float("inf"), dtype=torch.bfloat16, device="cuda")
    at = [int(c.st.seg_tok_start[int(c.st.prompt_seg_off[b])]) for b in range(2)]      # first tokens of the preambles
    for b in range(2):
        t["V"][at[b] + 5, :, 3], t["V"][at[b] + 70, :, 9], t["V"][at[b] + 100, :, 20] = x, -x, float("nan")
    c.call(ctx, c.plan(ctx), t)
    torch.cuda.synchronize()
    o = t["o"].float().cpu().numpy()
    for b, n in ((0, N), (1, N - 1)):
        mine = o[b, :n]
        assert (mine[..., 3] == np.inf).all() and (mine[..., 9] == -np.inf).all() and np.isnan(mine[..., 20]).all()
        rest = [e for e in range(heads[2]) if e not in (3, 9, 20)]
        assert np.isfinite(mine[..., rest]).all()


@pytest.mark.parametrize("score", [0.0, -20.0, -60.0, -80.0])
def test_an_infinite_value_of_little_weight(ctx, score):
    """down to weights of e^-80 (2^-116) of the largest an infinite V is infinite in the result"""
    d = 64
    c = TreeCase("bf16", 2, 2, d, 2, B=1, paths=1, k=0, preamble=200, resp=(40, 40), seed=6, n_nodes=[2])
    c.q[:] = 0.0
    c.q[..., 0] = 8.0
    c.K[:], c.Kr[:], c.kn[:] = 0.0, 0.0, 0.0
    c.K[10, :, 0] = score                                   # times 8 / sqrt(64)
    t = c.upload()
    t["V"][10] = float("inf")
    c.call(ctx, c.plan(ctx), t)
    torch.cuda.synchronize()
    assert (t["o"] == float("inf")).all()
