"""sp_tree_decode with infinities and NaN in V where the list of keys ends: whatever part of a step the last keys fill, whichever waves
take them and however the list is cut, they reach the rows that see them and no others."""
import gc

import numpy as np
import pytest
import torch

from oracle import sp_oracle_tree as ort
from paper_2404_06910_amd import binding as B

from tree_util import TreeCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


# (heads, nodes, prompts): one tile of rows; two tiles; waves for rows; a launch that has no groups of keys
SHAPES = [((4, 4, 64), 5, 1), ((8, 2, 128), 7, 2), ((8, 2, 128), 12, 1), ((20, 1, 64), 40, 2), ((8, 8, 128), 3, 80)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,N,prompts", SHAPES, ids=lambda x: str(x))
@pytest.mark.parametrize("left", [1, 15, 16, 17, 31, 0])
@pytest.mark.parametrize("whole", [1, 18])
def test_where_the_list_ends(ctx, dtype, heads, N, prompts, left, whole):
    """`left` keys in the last step of 32 behind `whole` steps or more; 18: lists that are cut where prompts are few"""
    total = 32 * max(whole, (N + 12) // 32 + 1) + left
    resp = 4
    c = TreeCase(dtype, *heads, N, B=prompts, paths=1, doc=(1, 1), query=1, k=0, preamble=total - N - resp, resp=(resp, resp), seed=left,
                 bias=N == 7, n_nodes=[N] * prompts)
    c.q *= 0.25                                             # scores of a few units: no weight is too small for a float
    inf, nan = np.inf, np.nan
    for b in (0, prompts - 1):
        c.Vr[b, resp - 1, :, 3], c.Vr[b, resp - 1, :, 4] = inf, nan
        c.vn[b, 1, :, 0], c.vn[b, 1, :, 1], c.vn[b, 1, :, 2] = inf, -inf, nan
        c.vn[b, N - 1, :, 5], c.vn[b, N - 1, :, 6] = -inf, nan
    t = c.upload()
    print("case:", dtype, heads, N, prompts, left, whole, flush=True)
    c.call(ctx, c.plan(ctx), t)
    torch.cuda.synchronize()
    got = t["o"].float().cpu().numpy()
    eps = 2.0 ** -24
    for b in (0, prompts - 1):
        K, V, pos = c.old_keys(b)
        assert (len(K) + N) % 32 == left
        with np.errstate(invalid="ignore"):
            o, absum, big = ort.tree_attention(c.q[b], c.kn[b], c.vn[b], K, V, c.parent[b], c.scale, c.slopes,
                                               None if c.new_pos is None else c.new_pos[b], pos)
        assert np.isfinite(o[..., 7:]).all() and (o[..., 3] == inf).all() and np.isnan(o[..., 4]).all()
        fine = np.isfinite(o)
        assert np.array_equal(np.isnan(o), np.isnan(got[b])) and np.array_equal(o[~fine & ~np.isnan(o)], got[b][~fine & ~np.isnan(o)])
        # as in TreeCase.check
        tol = absum * eps * (2 * (heads[2] + 8) * 1.45 * big[..., None] + 2 * (len(K) + N) + 16)
        if dtype == "bf16":
            tol = tol + 2.0 ** -8 * (absum + np.abs(o))
        assert (np.abs(got[b][fine] - o[fine]) <= tol[fine]).all()
