"""Scratch of cut tree launches: as many captures as a program makes, and launches of all sizes under one plan."""
import gc

import numpy as np
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


def test_hundreds_of_captures_under_one_plan(ctx):
    """each has scratch of its own, of what it needs; none is refused"""
    c = TreeCase("bf16", 4, 1, 128, 2, preamble=1500, resp=(40, 90), seed=1, n_nodes=[2, 2])
    plan, t = c.plan(ctx), c.upload()
    c.call(ctx, plan, t)
    torch.cuda.synchronize()
    c.check(t)
    want = t["o"].clone()
    main = torch.cuda.current_stream().cuda_stream
    graphs, free = [], torch.cuda.mem_get_info()[0]
    pool = torch.cuda.graph_pool_handle()
    for i in range(300):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            ctx.sp_set_stream(torch.cuda.current_stream().cuda_stream)
            c.call(ctx, plan, t)
        ctx.sp_set_stream(main)
        graphs.append(g)
    assert free - torch.cuda.mem_get_info()[0] < 300 * (4 << 20)
    for rep in range(2):
        for i in (0, 1, 128, 255, 256, 257, 299):
            t["o"].fill_(7.0)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(t["o"], want), i
    del graphs, g
    gc.collect()
    torch.cuda.synchronize()
    plan.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_launches_of_all_sizes(ctx, dtype):
    """few nodes, many, few again, on two streams, eager and captured, and after an update of the plan: every time with room enough"""
    c = TreeCase(dtype, 16, 2, 128, 64, preamble=1200, resp=(40, 90), seed=2, n_nodes=[64, 64])
    plan = c.plan(ctx)
    sizes = [1, 5, 64, 2, 33, 64, 1]

    def cut(N):                                             # the case with its first N nodes
        d = TreeCase.__new__(TreeCase)
        d.__dict__.update(c.__dict__)
        d.N, d.n_nodes = N, np.array([N, N], np.int32)
        for n in ("q", "kn", "vn", "parent"):
            setattr(d, n, np.ascontiguousarray(getattr(c, n)[:, :N]))
        return d

    main, side = torch.cuda.current_stream(), torch.cuda.Stream()
    for rep in range(2):
        cases = [cut(N) for N in sizes]
        eager, other, captured = ([d.upload() for d in cases] for _ in range(3))
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.sp_set_stream(torch.cuda.current_stream().cuda_stream)
            for d, t in zip(cases, captured):
                d.call(ctx, plan, t)
        for d, t, u in zip(cases, eager, other):
            ctx.sp_set_stream(main.cuda_stream)
            d.call(ctx, plan, t)
            ctx.sp_set_stream(side.cuda_stream)
            d.call(ctx, plan, u)
        ctx.sp_set_stream(main.cuda_stream)
        for _ in range(3):
            g.replay()
        torch.cuda.synchronize()
        for d, *ts in zip(cases, eager, other, captured):
            for t in ts:
                d.check(t)
            assert torch.equal(ts[0]["o"], ts[1]["o"]) and torch.equal(ts[0]["o"], ts[2]["o"])
        del g
        st = c.st
        plan.update(st.prompt_seg_off, st.seg_tok_start, st.seg_tok_len, st.seg_parent, st.seg_path, st.n_tokens)
    plan.close()
