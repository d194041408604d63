"""What a launch can hold: sizes beyond it are refused before anything runs, and the widest group of heads is not."""
import gc
import math

import numpy as np
import pytest
import torch

from oracle import sp_oracle_tree as ort
from paper_2404_06910_amd import binding as B

from gpu_util import TORCH_DT, SP_DT, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()
    c.close()


def test_more_workgroups_than_a_launch_has(ctx):
    prompts, heads = 1 << 16, 128                           # 2^23 pairs
    i = np.arange(prompts + 1, dtype=np.int32)
    none = np.full(prompts, -1, np.int32)
    plan = B.Plan(ctx, i, i[:-1], np.ones(prompts, np.int32), none, none, prompts, heads, heads, 64, B.SP_BF16)
    x = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    p, q = x.data_ptr(), x.data_ptr() + 64                  # refused before anybody reads or writes there
    st = B.lib().sp_tree_decode(ctx._h, plan._h, None, 0, p, p, heads * 64, 64, p, p, None, 1, None, 0, None, None, 1, None, p, p, p, q, 1.0)
    assert st == -3 and b"2^23" in B.lib().sp_last_error(ctx._h)
    z = torch.zeros(64, dtype=torch.int32, device="cuda").data_ptr()
    st = B.lib().sp_tree_accept(ctx._h, 1 << 24, 1, None, None, z, z, B.SP_BF16, 1, 0, 1, 64, p, q, None, 1, None, 0, z, z, z, z)
    assert st == -3 and b"2^24" in B.lib().sp_last_error(ctx._h)
    plan.close()
    torch.cuda.synchronize()
    assert (x == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_widest_group_of_heads(ctx, dtype):
    """65535 query heads on one KV head, 64 nodes: 4 194 240 rows of one prompt"""
    H, N, d, P = 65535, 64, 64, 5
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(TORCH_DT[dtype])
    one = lambda v: np.array([v], np.int32)
    plan = B.Plan(ctx, np.array([0, 1], np.int32), one(0), one(P), one(-1), one(-1), P, H, 1, d, SP_DT[dtype])
    K, V, kn, vn, q = r(P, 1, d), r(P, 1, d), r(1, N, 1, d), r(1, N, 1, d), r(1, N, H, d)
    Kr, Vr, o = r(1, N, 1, d), r(1, N, 1, d), torch.full_like(q, 7.0)
    parent = np.array([[(i - 1) // 2 if i else -1 for i in range(N)]], np.int32)
    scale = 1 / math.sqrt(d)
    print("case:", dtype, flush=True)
    ctx.sp_tree_decode(plan, None, 0, K, V, Kr, Vr, N, q, kn, vn, o, scale, parent=dev(parent))
    torch.cuda.synchronize()
    host = lambda t: t.float().cpu().numpy()
    which = [0, 1, 32767, 32768, 65533, 65534]
    ref, absum, big = ort.tree_attention(host(q[0][:, which]), host(kn[0]), host(vn[0]), host(K), host(V), parent[0], scale)
    eps = 2.0 ** -24                                        # as in TreeCase.check
    tol = absum * eps * (2 * (d + 8) * 1.45 * big[..., None] + 2 * (P + N) + 16)
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (absum + np.abs(ref))
    assert (np.abs(host(o[0][:, which]) - ref) <= tol).all()
    assert not (o == 7).all(dim=3).any() and torch.equal(Kr, kn) and torch.equal(Vr, vn)
    plan.close()
