"""sp_tree_decode against the 64-bit oracle: types, head layouts, lengths, trees, what is left alone, refusals, graphs, streams."""
import gc

import numpy as np
import pytest
import torch

from paper_2404_06910_amd import binding as B

from gpu_util import dev
from tree_util import TreeCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()                                            # plans in reference cycles go now, and not in some later capture
    c.close()


def _run(ctx, c, **kw):
    t = c.upload()
    plan = c.plan(ctx)
    c.call(ctx, plan, t, **kw)
    torch.cuda.synchronize()
    return t


HEADS = [(4, 4, 64), (8, 8, 128), (8, 2, 128), (6, 2, 64), (7, 1, 128), (16, 2, 64), (20, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d-%d-%d" % h)
@pytest.mark.parametrize("N", [1, 2, 5, 16, 33, 64])
@pytest.mark.parametrize("bias", [False, True], ids=["", "bias"])
def test_shapes(ctx, dtype, heads, N, bias):
    c = TreeCase(dtype, *heads, N, bias=bias, seed=N + 100 * bias, n_nodes=[N, max(1, N - 3)])
    print("case:", dtype, heads, N, bias, flush=True)
    c.check(_run(ctx, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("keys", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 500, 1111])
def test_lengths(ctx, dtype, keys):
    """cached keys around the tile sizes, and one document or a long response to hold them"""
    for resp in (False, True):
        kw = dict(preamble=1, doc=(1, 1), resp=(keys, keys)) if resp else dict(preamble=keys, doc=(1, 1), resp=(0, 0))
        c = TreeCase(dtype, 4, 2, 128, 7, paths=1, query=1, k=0, seed=keys, n_nodes=[7, 4], **kw)
        print("case:", dtype, keys, resp, flush=True)
        c.check(_run(ctx, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k", [0, 1, 4, 9])
@pytest.mark.parametrize("packing", ["interleaved", "grouped"])
def test_kept_paths(ctx, dtype, k, packing):
    c = TreeCase(dtype, 8, 2, 64, 9, B=3, paths=9, k=k, packing=packing, doc=(1, 30), seed=k)
    if k > 1:
        c.kept[1, 1:] = -1                                  # entries below zero are none
    keep = c.kept
    t = _run(ctx, c)
    c.kept = [[j for j in row if j >= 0] for row in keep]
    c.check(t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_major_cache_and_padded_strides(ctx, dtype):
    c = TreeCase(dtype, 8, 4, 128, 12, seed=5)
    for layout in ("head", "padded"):
        t = c.upload()
        for n in ("K", "V"):
            x = t[n]
            if layout == "head":
                t[n] = x.transpose(0, 1).contiguous().transpose(0, 1)
            else:
                wide = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + 8), float("nan"), dtype=x.dtype, device="cuda")
                wide[:, :-1, :-8] = x
                t[n] = wide[:, :-1, :-8]
        c.call(ctx, c.plan(ctx), t)
        torch.cuda.synchronize()
        c.check(t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_defaults(ctx, dtype):
    """no parent table: a chain; no node counts: all; no lengths: an empty response cache, or resp_len_add rows of it"""
    c = TreeCase(dtype, 4, 2, 64, 10, resp=(0, 0), seed=6, room=8)
    chain = np.tile(np.arange(-1, 9, dtype=np.int32), (2, 1))
    for add in (0, 5):
        t = _run(ctx, c, parent=None, n_nodes=None, resp_len=None, resp_len_add=add)
        c.check(t, n_nodes=[10, 10], parent=chain, lengths=[add, add])
    t = _run(ctx, c, parent=None, resp_len=dev(np.array([3, 0], np.int32)), resp_len_add=2)
    c.check(t, parent=chain, lengths=[5, 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tables_out_of_contract(ctx, dtype):
    """parents that do not come before count as none; node counts are clamped; rows beyond the cache are dropped"""
    c = TreeCase(dtype, 4, 4, 64, 6, B=4, resp=(4, 4), room=0, seed=7)
    bad = np.array([[0, 1, 0, 7, -9, 3], [-1, 0, 2, 2, 1 << 30, -(1 << 31)], [-1, 0, 1, 2, 3, 4], [-1, 0, 0, 0, 0, 0]], np.int32)
    good = np.array([[-1, -1, 0, -1, -1, 3], [-1, 0, -1, 2, -1, -1], [-1, 0, 1, 2, 3, 4], [-1, 0, 0, 0, 0, 0]], np.int32)
    t = _run(ctx, c, parent=dev(bad), n_nodes=dev(np.array([6, 99, -3, 1 << 30], np.int32)))
    c.check(t, n_nodes=[6, 6, 0, 6], parent=good)
    for lengths in ([7, 9, 10, 25], [0, 8, 10, 11]):        # the cache has 10 rows
        t = _run(ctx, c, n_nodes=None, resp_len=dev(np.array(lengths, np.int32)))
        c.check(t, n_nodes=[6] * 4, lengths=lengths)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_take_no_part_may_hold_anything(ctx, dtype):
    """infinities and NaN in response rows behind the response, in nodes that are not there and in tokens of other paths"""
    c = TreeCase(dtype, 8, 2, 128, 13, seed=8, resp=(3, 9), n_nodes=[5, 9])
    clean = _run(ctx, c)
    t = c.upload()
    seen = np.zeros(c.st.n_tokens, bool)
    for b in range(c.B):
        from oracle import sp_oracle as orc
        seen[orc.joined_cache_index(c.st.prompt_seg_off, c.st.seg_tok_start, c.st.seg_tok_len, c.st.seg_path, b, c.kept[b])] = True
        for n, v in (("Kr", float("nan")), ("Vr", float("inf"))):
            t[n][b, int(c.resp_len[b]):] = v
        for n, v in (("kn", float("nan")), ("vn", float("-inf")), ("q", float("nan"))):
            t[n][b, int(c.n_nodes[b]):] = v
    t["K"][dev(~seen)], t["V"][dev(~seen)] = float("nan"), float("inf")
    c.call(ctx, c.plan(ctx), t)
    torch.cuda.synchronize()
    assert torch.equal(t["o"], clean["o"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_reach_only_who_sees_them(ctx, dtype):
    """a brother's V of infinity has weight zero and must not make NaN of it"""
    c = TreeCase(dtype, 4, 2, 64, 5, B=1, seed=9, n_nodes=[5])
    c.parent = np.array([[-1, 0, 0, 1, 2]], np.int32)
    t = c.upload()
    t["vn"][0, 1] = float("inf")
    c.call(ctx, c.plan(ctx), t)
    torch.cuda.synchronize()
    o = t["o"].float().cpu().numpy()[0]
    assert np.isfinite(o[[0, 2, 4]]).all() and (o[[1, 3]] == np.inf).all()


def test_equal_calls_are_equal_on_streams_and_in_graphs(ctx):
    c = TreeCase("bf16", 8, 2, 128, 21, B=2, preamble=300, resp=(40, 90), seed=10, n_nodes=[21, 17])
    plan = c.plan(ctx)
    t = c.upload()
    c.call(ctx, plan, t)
    torch.cuda.synchronize()
    c.check(t)
    want = t["o"].clone()
    main = torch.cuda.current_stream().cuda_stream
    sides = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in sides:                                          # two launches that may overlap
        u = dict(t, o=torch.full_like(t["o"], 7.0), Kr=t["Kr"].clone(), Vr=t["Vr"].clone())
        outs.append(u)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, u in zip(sides, outs):
            ctx.sp_set_stream(s.cuda_stream)
            c.call(ctx, plan, u)
    ctx.sp_set_stream(main)
    torch.cuda.synchronize()
    assert all(torch.equal(u["o"], want) for u in outs)
    graphs = []
    for u in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.sp_set_stream(torch.cuda.current_stream().cuda_stream)
            c.call(ctx, plan, u)
        ctx.sp_set_stream(main)
        graphs.append(g)
    for rep in range(4):
        for u in outs:
            u["o"].fill_(7.0)
        t["q"].mul_(-1.0)
        c.call(ctx, plan, t)
        torch.cuda.synchronize()
        want = t["o"].clone()
        for g, s in zip(graphs, sides):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u["o"], want) for u in outs), rep


def test_large_offsets(ctx):
    """a response cache whose last prompt lies behind element 2^31, and keys of the packed cache behind 4 GB"""
    c = TreeCase("bf16", 8, 8, 128, 3, B=2, k=1, resp=(5, 5), seed=11, n_nodes=[3, 3])
    t = c.upload()
    rows, heads, d = 1, 8, 128
    cap = (1 << 31) // (heads * d) + 16                      # prompt 1 begins behind 2^31 elements
    old = c.cap
    big = {}
    for n in ("Kr", "Vr"):
        x = torch.empty((2, cap, heads, d), dtype=torch.bfloat16, device="cuda")
        x[:, :old] = t[n]
        big[n] = x
    stride = (1 << 31) // c.st.n_tokens // 8 * 8             # tokens far apart: the last one behind 4 GB
    for n in ("K", "V"):
        flat = torch.empty(stride * (c.st.n_tokens - 1) + heads * d, dtype=torch.bfloat16, device="cuda")
        view = torch.as_strided(flat, (c.st.n_tokens, heads, d), (stride, d, 1))
        view.copy_(t[n])
        big[n] = view
    plan = c.plan(ctx)
    ctx.sp_tree_decode(plan, t["kept"], c.k, big["K"], big["V"], big["Kr"], big["Vr"], cap, t["q"], t["kn"], t["vn"], t["o"], c.scale,
                       parent=t["parent"], n_nodes=t["n_nodes"], resp_len=t["resp_len"])
    torch.cuda.synchronize()
    t["Kr"], t["Vr"] = big["Kr"][:, :old], big["Vr"][:, :old]
    c.check(t)


def test_refusals(ctx):
    c = TreeCase("bf16", 4, 2, 64, 5, seed=12)
    plan = c.plan(ctx)
    t = c.upload()

    def status(**kw):
        u = dict(t)
        args = {n: kw.pop(n) for n in list(kw) if n not in u}
        u.update(kw)
        with pytest.raises((B.SpError, ValueError)) as e:
            c.call(ctx, plan, u, **args)
        return getattr(e.value, "status", None)

    wide = lambda n, N: torch.zeros((c.B, N) + tuple(t[n].shape[2:]), dtype=torch.bfloat16, device="cuda")
    assert status(q=wide("q", 65), o=wide("q", 65), kn=wide("kn", 65), vn=wide("vn", 65), parent=None) == -3
    assert status(o=t["q"]) == -1
    assert status(resp_len_add=-1) == -1
    assert status(q=t["q"].cpu()) is None and status(q=t["q"].float()) is None
    assert status(parent=t["parent"].long()) is None and status(parent=t["parent"][:, :4].contiguous()) is None
    assert status(q=t["q"].transpose(1, 2)) is None and status(n_nodes=t["n_nodes"][:1]) is None
    empty = lambda n: torch.zeros((c.B, 0) + tuple(t[n].shape[2:]), dtype=torch.bfloat16, device="cuda")
    assert status(q=empty("q"), o=empty("q"), kn=empty("kn"), vn=empty("vn"), parent=None) == -1
    bias = TreeCase("bf16", 4, 2, 64, 5, seed=12, bias=True)
    bplan, bt = bias.plan(ctx), bias.upload()
    for missing in ("pos_resp", "new_pos"):
        with pytest.raises(B.SpError) as e:
            bias.call(ctx, bplan, bt, **{missing: None})
        assert e.value.status == -1
    other = B.Context(0)
    with pytest.raises(B.SpError):
        c.call(other, plan, t)
    other.close()
    torch.cuda.synchronize()
    assert (t["o"] == 7).all()                               # nothing ran
