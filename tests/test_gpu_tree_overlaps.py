"""Memory that the results of the generation loop's calls may not share: parts of inputs, and other results."""
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


def _refused(call):
    with pytest.raises(B.SpError) as e:
        call()
    torch.cuda.synchronize()
    return e.value.status == -1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_results_on_a_part_of_the_nodes(ctx, dtype):
    c = TreeCase(dtype, 4, 4, 64, 6, seed=1, n_nodes=[6, 6])
    plan, t = c.plan(ctx), c.upload()
    n = t["q"].numel()
    whole = torch.zeros(2 * n, dtype=t["q"].dtype, device="cuda")
    at = lambda first: whole[first:first + n].view(t["q"].shape)
    for name in ("q", "kn", "vn"):
        for first in (64, n - 64):                          # a head of the other, before and behind
            assert _refused(lambda: c.call(ctx, plan, dict(t, **{name: at(0), "o": at(first)})))
            assert _refused(lambda: c.call(ctx, plan, dict(t, **{name: at(first), "o": at(0)})))
    assert (whole == 0).all()
    beside = dict(t, q=at(0), o=at(n))
    beside["q"].copy_(t["q"])
    c.call(ctx, plan, beside)
    torch.cuda.synchronize()
    beside["o"] = beside["o"].clone()
    c.check(beside)


def test_token_and_logprob(ctx):
    x, u = torch.zeros((4, 64), device="cuda"), torch.zeros(4, device="cuda")
    both = torch.zeros(7, dtype=torch.int32, device="cuda")
    for a, b in ((both[:4], both[:4]), (both[:4], both[3:]), (both[3:], both[:4])):
        assert _refused(lambda: ctx.sp_sample(x, u, a, b.view(torch.float32)))
    eight = torch.full((8,), -7, dtype=torch.int32, device="cuda")
    ctx.sp_sample(x, u, eight[:4], eight[4:].view(torch.float32))
    torch.cuda.synchronize()
    assert (eight[:4] == 0).all()


def test_results_of_an_acceptance(ctx):
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    K, V = (torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos = torch.zeros((2, 8), device="cuda")
    x = dict(draft=z(2, 4), sampled=z(2, 4), path=z(2, 4), n_accepted=z(2), next_token=z(2), resp_len_out=z(2), parent=z(2, 4), n_nodes=z(2),
             resp_len=z(2), pos_resp=pos, K_resp=K, V_resp=V)

    def refused(**kw):
        return _refused(lambda: ctx.sp_tree_accept(**dict(x, **kw)))

    for a in ("n_accepted", "next_token", "resp_len_out"):
        assert refused(**{a: x["path"].view(-1)[1:3]}) and refused(**{a: pos.view(torch.int32).view(-1)[3:5]})
        for b in ("n_accepted", "next_token", "resp_len_out"):
            assert a == b or refused(**{a: x[b]})
    assert refused(next_token=x["resp_len"], resp_len_out=x["resp_len"])
    table = torch.zeros((2, 8), device="cuda")
    for name in ("draft", "sampled", "parent", "path"):
        assert refused(pos_resp=table, **{name: table.view(torch.int32)[1:].view(2, 4)})
    ctx.sp_tree_accept(**dict(x, resp_len_out=x["resp_len"]))
    torch.cuda.synchronize()
