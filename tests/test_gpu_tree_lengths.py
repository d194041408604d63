"""sp_tree_decode with response lengths far beyond the cache, up to the largest that there are: its rows take part, and no node is stored."""
import gc

import numpy as np
import pytest
import torch

from paper_2404_06910_amd import binding as B

from gpu_util import dev
from tree_util import TreeCase

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


def _case(dtype, bias):
    return TreeCase(dtype, 4, 2, 64, 64, B=4, resp=(6, 6), bias=bias, seed=13, n_nodes=[64, 64, 5, 64])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [False, True], ids=["", "bias"])
def test_lengths_up_to_the_largest(ctx, dtype, bias):
    """length + node passes 2^31 for some of the nodes, or all but the first"""
    c = _case(dtype, bias)
    lengths = [MOST, MOST - 62, MOST - 63, 1 << 30]
    t = c.upload()
    print("case:", dtype, bias, flush=True)
    c.call(ctx, c.plan(ctx), t, resp_len=dev(np.array(lengths, np.int32)))
    torch.cuda.synchronize()
    c.check(t, lengths=lengths)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_length_for_all_prompts(ctx, dtype):
    c = _case(dtype, False)
    for add in (MOST, MOST - 1, MOST - 63):
        t = c.upload()
        print("case:", dtype, add, flush=True)
        c.call(ctx, c.plan(ctx), t, resp_len=None, resp_len_add=add)
        torch.cuda.synchronize()
        c.check(t, lengths=[add] * 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_last_rows_of_the_cache(ctx, dtype):
    """nodes for which there is room are stored, those behind them are not"""
    c = _case(dtype, True)
    lengths = [c.cap - 1, c.cap, c.cap - 30, c.cap - 64]
    t = c.upload()
    c.call(ctx, c.plan(ctx), t, resp_len=dev(np.array(lengths, np.int32)))
    torch.cuda.synchronize()
    c.check(t, lengths=lengths)
