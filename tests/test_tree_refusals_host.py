"""Refusals that need no GPU: calls without a context, and what the binding checks before the library is called."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2404_06910_amd import binding as B


def test_calls_without_a_context():
    L = B.lib()
    n = None
    assert L.sp_tree_decode(n, n, n, 0, n, n, 0, 0, n, n, n, 1, n, 0, n, n, 1, n, n, n, n, n, 1.0) == -1
    assert b"ctx" in L.sp_last_error(None)
    assert L.sp_sample(n, n, 0, 1, 1, 4, 1, n, n, n, n, n, n, n) == -1
    assert L.sp_tree_accept(n, 1, 1, n, n, n, n, 0, 1, 0, 1, 64, n, n, n, 1, n, 0, n, n, n, n) == -1


class _NoContext(B.Context):
    def __init__(self):
        self._h = C.c_void_p()


@pytest.fixture
def ctx():
    return _NoContext()


class _Plan:
    _h, dtype, n_prompts, n_tokens, n_q_heads, n_kv_heads, head_dim = C.c_void_p(), B.SP_F32, 2, 9, 4, 2, 64


def test_binding_checks(ctx):
    z, i = torch.zeros, lambda *s: torch.zeros(s, dtype=torch.int32)
    kv, new, q = z(9, 2, 64), z(2, 3, 2, 64), z(2, 3, 4, 64)
    resp = z(2, 8, 2, 64)

    def tree(K=kv, V=kv, q=q, k=new, v=new, o=q, cap=8, kept=i(2, 1), **kw):
        ctx.sp_tree_decode(_Plan, kept, 1, K, V, resp, resp.clone(), cap, q, k, v, o, 1.0, **kw)

    for kw, word in ((dict(V=kv.transpose(0, 1)), "strides"), (dict(o=z(2, 3, 4, 32)), "o_out"), (dict(q=z(3, 3, 4, 64)), "n_prompts"),
                     (dict(k=z(2, 4, 2, 64)), "k_new"), (dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), "contiguous"),
                     (dict(q=q.bfloat16(), o=q.bfloat16()), "dtype"), (dict(), "CUDA"),
                     (dict(q=z(2, 3, 2, 64), o=z(2, 3, 2, 64)), "n_q_heads"), (dict(k=z(2, 3, 1, 64), v=z(2, 3, 1, 64)), "n_kv_heads"),
                     (dict(K=kv[:8], V=kv[:8]), "n_tokens"), (dict(cap=9), "resp_capacity"), (dict(q=q[0], o=q[0]), "max_nodes")):
        with pytest.raises(ValueError, match=word):
            tree(**kw)
    with pytest.raises(ValueError, match="inner stride"):
        ctx.sp_sample(z(4, 8).t(), z(8), i(8))
    with pytest.raises(ValueError, match="CUDA"):
        ctx.sp_sample(z(4, 8), z(4), i(4))
    with pytest.raises(ValueError, match="alike"):
        ctx.sp_tree_accept(i(2, 3), i(2, 3), resp, z(2, 7, 2, 64), i(2, 3), i(2), i(2), i(2))
    with pytest.raises(ValueError, match="contiguous"):
        ctx.sp_tree_accept(i(2, 3), i(2, 3), resp.transpose(1, 2), resp.transpose(1, 2), i(2, 3), i(2), i(2), i(2))
    for t, n in ((i(3), 2), (i(4)[::2], 2), (z(2), 2), (np.int32, None)):
        if isinstance(t, torch.Tensor):
            with pytest.raises(ValueError):
                B._i32_dev(t, "t", n)
    assert B._i32_dev(None, "t", 5) is None
