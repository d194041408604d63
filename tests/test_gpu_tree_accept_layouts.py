"""sp_tree_accept on caches whose extents of 1 have strides of their own: one KV head kept head by head, one prompt of a larger cache."""
import gc

import numpy as np
import pytest
import torch

from paper_2404_06910_amd import binding as B

from gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


def _accept(ctx, K, V):
    """a tree of four nodes of which 0 and 3 are taken: row len + 3 goes to len + 1"""
    prompts = K.shape[-4]
    i = lambda a: dev(np.tile(np.array(a, np.int32), (prompts, 1)))
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    path, n, nxt, out = z(prompts, 4), z(prompts), z(prompts), z(prompts)
    ctx.sp_tree_accept(i([0, 5, 6, 7]), i([7, 1, 1, 9]), K, V, path, n, nxt, out, parent=i([-1, 0, 0, 0]), resp_len_add=2)
    torch.cuda.synchronize()
    assert (n == 2).all() and (nxt == 9).all() and (out == 4).all() and (path == torch.tensor([0, 3, -1, -1], device="cuda")).all()


@pytest.mark.parametrize("layers", [0, 3])
@pytest.mark.parametrize("prompts", [1, 2])
def test_one_head_kept_head_by_head(ctx, layers, prompts):
    lead = (layers, prompts) if layers else (prompts,)
    store = [torch.randn(lead + (1, 8, 64), device="cuda") for _ in range(2)]        # heads, then rows
    K, V = (x.transpose(-3, -2) for x in store)
    want = [x.clone() for x in store]
    for x in want:
        x[..., 0, 3, :] = x[..., 0, 5, :]
    _accept(ctx, K, V)
    assert torch.equal(store[0], want[0]) and torch.equal(store[1], want[1])


def test_one_prompt_of_a_larger_cache(ctx):
    store = [torch.randn((3, 4, 8, 2, 64), device="cuda") for _ in range(2)]
    K, V = (x[:, 2:3] for x in store)
    want = [x.clone() for x in store]
    for x in want:
        x[:, 2, 3] = x[:, 2, 5]
    _accept(ctx, K, V)
    assert torch.equal(store[0], want[0]) and torch.equal(store[1], want[1])


def test_blocks_that_are_not_contiguous_are_refused(ctx):
    z = lambda *shape: torch.zeros(shape, device="cuda")
    for make in (lambda: z(3, 2, 2, 8, 64).transpose(2, 3), lambda: z(2, 3, 8, 2, 64).transpose(0, 1), lambda: z(2, 8, 2, 128)[..., :64]):
        with pytest.raises(ValueError, match="contiguous"):
            _accept(ctx, make(), make())
