"""What calls of the generation loop share: scratch that one plan leaves to the next, and memory that a result may not share with an input."""
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
    gc.collect()
    c.close()


def test_scratch_of_a_plan_that_is_gone(ctx):
    """A plan goes while its launches wait on one stream; another plan, made before, needs scratch on another stream meanwhile."""
    main, side = torch.cuda.current_stream(), torch.cuda.Stream()
    cases = [TreeCase("bf16", 8, 2, 128, 20, preamble=900 + 200 * i, resp=(40, 90), seed=i, n_nodes=[20, 13]) for i in range(2)]
    slow = torch.randn(4096, 4096, device="cuda")
    for rep in range(3):
        t = [c.upload() for c in cases]
        plans = [c.plan(ctx) for c in cases]
        torch.cuda.synchronize()
        for _ in range(8):
            slow = (slow @ slow).clamp_(-1, 1)              # some milliseconds before the first plan's launches
        for _ in range(4):
            cases[0].call(ctx, plans[0], t[0])
        plans[0].close()
        ctx.sp_set_stream(side.cuda_stream)
        for _ in range(4):
            cases[1].call(ctx, plans[1], t[1])
        ctx.sp_set_stream(main.cuda_stream)
        torch.cuda.synchronize()
        plans[1].close()
        for c, x in zip(cases, t):
            c.check(x)


def test_scratch_goes_round(ctx):
    """plans that come and go, on one stream and captured, do not pile up memory"""
    c = TreeCase("bf16", 8, 2, 128, 20, preamble=900, resp=(40, 90), seed=5, n_nodes=[20, 13])
    t = c.upload()
    free = []
    for rep in range(24):
        plan = c.plan(ctx)
        main = torch.cuda.current_stream().cuda_stream
        ctx.sp_set_stream(main)
        c.call(ctx, plan, t)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.sp_set_stream(torch.cuda.current_stream().cuda_stream)
            c.call(ctx, plan, t)
        ctx.sp_set_stream(main)
        t["o"].fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        c.check(t, prompts=[rep % 2])
        plan.close()
        del g
        free.append(torch.cuda.mem_get_info()[0])
    assert free[4] - free[-1] < 64 << 20, free              # 20 rounds at 16 or 32 MiB would be more


def test_results_on_inputs_are_refused(ctx):
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    K, V = (torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = dict(draft=z(2, 4), sampled=z(2, 4), path=z(2, 4), n_accepted=z(2), next_token=z(2), resp_len_out=z(2), parent=z(2, 4), n_nodes=z(2),
             resp_len=z(2))

    def refused(**kw):
        a = dict(x, K_resp=K, V_resp=V)
        a.update(kw)
        with pytest.raises(B.SpError) as e:
            ctx.sp_tree_accept(**a)
        return e.value.status == -1

    for wide in ("draft", "sampled", "parent"):
        assert refused(path=x[wide]) and refused(next_token=x[wide][0, 2:])
    for narrow in ("n_nodes", "resp_len"):
        assert refused(n_accepted=x[narrow]) and refused(next_token=x[narrow])
    assert refused(resp_len_out=x["n_nodes"]) and refused(V_resp=K)

    logits, u, token = torch.zeros((4, 64), device="cuda"), torch.zeros(4, device="cuda"), z(4)
    for kw in (dict(logprob=u), dict(top_k=token), dict(temperature=u, logprob=u), dict(logprob=logits[1, 8:12])):
        with pytest.raises(B.SpError) as e:
            ctx.sp_sample(logits, kw.get("temperature", u) + 0 if "temperature" in kw else u, token, **kw)
        assert e.value.status == -1
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [50, 3001, 60001])
def test_settings_without_bound(ctx, dtype, vocab):
    """an infinite temperature weighs all tokens alike, except beside an infinite logit; neither leaves a row without a token"""
    x = torch.randn((4, -(-vocab // 8) * 8), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)[:, :vocab]
    x[2:, vocab // 2] = float("inf")
    x[:, 0] = float("-inf")
    u = dev(np.array([0.0, 0.999999, 0.3, 0.9], np.float32))
    inf = torch.full((4,), float("inf"), device="cuda")
    token, logprob = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    for min_p in (None, torch.full((4,), 0.5, device="cuda")):
        ctx.sp_sample(x, u, token, logprob, temperature=inf, min_p=min_p)
        torch.cuda.synchronize()
        got, lp = token.cpu().numpy(), logprob.cpu().numpy()
        host = x.float().cpu().numpy()
        order = [np.argsort(-host[r], kind="stable") for r in range(2)]
        # weights are equal, and a running weight exceeds u of all of them at place floor(u n) of n
        assert list(got) == [order[0][0], order[1][int(float(u[1]) * (vocab - 1))], vocab // 2, vocab // 2]
        assert np.allclose(lp, [-np.log(vocab - 1)] * 2 + [0, 0], rtol=2.0 ** -22, atol=0)
