"""sp_sample of more rows than one launch can have workgroups."""
import gc

import pytest
import torch

from paper_2404_06910_amd import binding as B

from gpu_util import TORCH_DT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,per", [((1 << 21) + 1, (1 << 20) - 5), ((1 << 22) + 3, (1 << 20) - 5), ((1 << 22) + 3, (1 << 21) + 77),
                                      ((1 << 22) + 3, 1 << 30), ((1 << 22) + 3, 1 << 21)])
def test_rows_of_several_launches(ctx, dtype, rows, per):
    """against the definition in doubles, row by row on the device; settings change inside a launch and between two"""
    vocab = 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, vocab), generator=g, device="cuda").mul_(2).to(TORCH_DT[dtype])
    u = torch.rand(rows, generator=g, device="cuda")
    sets = -(-rows // per)
    T = torch.tensor([0.9, 0.5, 2.0, 0.0, 0.8][:sets], device="cuda")
    k = torch.tensor([0, 3, 8, 0, 2][:sets], dtype=torch.int32, device="cuda")
    token, logprob = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    print("case:", dtype, rows, per, flush=True)
    ctx.sp_sample(x, u, token, logprob, temperature=T, top_k=k, rows_per_set=per)
    torch.cuda.synchronize()
    each = torch.arange(rows, device="cuda") // per
    v, order = torch.sort(x.double(), dim=1, descending=True, stable=True)
    t, n = T.double()[each], torch.where(k > 0, k, vocab)[each]
    greedy = t <= 0
    z = (v - v[:, :1]) / torch.where(greedy, 1.0, t)[:, None]
    place = torch.arange(vocab, device="cuda")
    w = torch.exp(z) * (place < torch.where(greedy, 1, n)[:, None])
    run = torch.cumsum(w, 1)
    border = u.double()[:, None] * run[:, -1:]
    at = (run <= border).sum(1, keepdim=True).clamp(max=vocab - 1)
    # weights are multiples of 2^-59, sums of doubles end at 2^-50: nearer borders than 2^-45 are not told apart
    sure = ((run - border).abs() / run[:, -1:]).amin(1) > 2.0 ** -45
    assert sure.double().mean() > 0.999
    want = torch.gather(order, 1, at)[:, 0].int()
    assert torch.equal(token[sure], want[sure])
    lp = (torch.gather(z, 1, at) - torch.log(run[:, -1:]))[:, 0]
    lp[greedy] = 0
    assert ((logprob.double() - lp).abs()[sure] <= 2.0 ** -24 * lp.abs()[sure] + 2.0 ** -45).all()
