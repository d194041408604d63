"""sp_tree_decode where a launch has many workgroups: the other ways of sharing out rows and keys, against the 64-bit oracle."""
import gc

import pytest
import torch

from paper_2404_06910_amd import binding as B

from tree_util import TreeCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


# (prompts, heads, nodes): from fewer workgroups than compute units to several for each, with 16, 32, 64 and more rows to a KV head
MANY = [(24, (16, 16, 64), 7), (40, (16, 16, 128), 16), (20, (32, 16, 64), 16), (40, (16, 8, 64), 15), (70, (16, 8, 64), 12),
        (20, (16, 8, 64), 29), (40, (16, 8, 128), 32), (20, (16, 8, 64), 64), (12, (40, 8, 64), 33), (33, (64, 8, 64), 19),
        (9, (64, 8, 128), 64), (40, (64, 8, 64), 33)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [False, True], ids=["", "bias"])
@pytest.mark.parametrize("many", MANY, ids=lambda m: "%d-%d-%d-%d-%d" % (m[0], *m[1], m[2]))
def test_many_prompts(ctx, dtype, bias, many):
    n, heads, nodes = many
    c = TreeCase(dtype, *heads, nodes, B=n, bias=bias, resp=(0, 60), seed=n + nodes)
    print("case:", dtype, many, bias, flush=True)
    t = c.upload()
    c.call(ctx, c.plan(ctx), t)
    torch.cuda.synchronize()
    c.check(t, prompts=range(0, n, 5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k", [62, 63, 64, 70, 100])
def test_many_prompts_with_many_kept_paths(ctx, dtype, k):
    """a source of keys for every kept path, in workgroups that would be a single wave by their rows"""
    c = TreeCase(dtype, 16, 16, 64, 3, B=36, paths=100, k=k, doc=(1, 3), seed=k)
    print("case:", dtype, k, flush=True)
    t = c.upload()
    c.call(ctx, c.plan(ctx), t)
    torch.cuda.synchronize()
    c.check(t, prompts=range(0, 36, 7))
