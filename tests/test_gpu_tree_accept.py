"""sp_tree_accept against the oracle's walk, with every byte of the caches compared."""
import gc

import numpy as np
import pytest
import torch

from oracle import sp_oracle_tree as ort
from paper_2404_06910_amd import binding as B

from gpu_util import TORCH_DT, dev
from tree_util import random_parents

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    gc.collect()                                            # plans in reference cycles go now, and not in some later capture
    c.close()


class Case:
    def __init__(self, dtype, B_, N, layers, heads, d, cap, seed, agree=0.8, resp=None, chain=False, pos=True, pad=0):
        rng = np.random.default_rng(seed)
        self.rng, self.B, self.N, self.cap = rng, B_, N, cap
        self.parent = np.tile(np.arange(-1, N - 1, dtype=np.int32), (B_, 1)) if chain else random_parents(rng, B_, N)
        self.n_nodes = rng.integers(0, N + 1, B_).astype(np.int32)
        self.draft = rng.integers(0, 6, (B_, N)).astype(np.int32)
        self.sampled = rng.integers(0, 6, (B_, N)).astype(np.int32)
        for b in range(B_):                                  # most nodes agree with one of their children
            for i in range(N):
                ch = np.flatnonzero(self.parent[b] == i)
                if len(ch) and rng.random() < agree:
                    self.sampled[b, i] = self.draft[b, rng.choice(ch)]
        self.resp_len = (rng.integers(0, cap - N + 1, B_) if resp is None else np.asarray(resp)).astype(np.int32)
        dt = TORCH_DT[dtype]
        block = B_ * cap * heads * d
        whole = torch.randn((2, layers, block + pad), device="cuda").to(dt)
        self.whole = whole
        self.K, self.V = (torch.as_strided(whole[j], (layers, B_, cap, heads, d), (block + pad, cap * heads * d, heads * d, d, 1))
                          for j in range(2))
        self.pos = torch.rand((B_, cap), device="cuda") if pos else None
        self.before = whole.clone(), None if self.pos is None else self.pos.clone()
        self.out = [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((B_, N), (B_,), (B_,), (B_,))]

    def call(self, ctx, in_place=False, **kw):
        lens = dev(self.resp_len)
        args = dict(parent=dev(self.parent), n_nodes=dev(self.n_nodes), resp_len=lens, pos_resp=self.pos)
        args.update(kw)
        path, count, nxt, out = self.out
        if in_place:
            out = self.out[3] = lens
        one = self.K.shape[0] == 1
        ctx.sp_tree_accept(dev(self.draft), dev(self.sampled), self.K[0] if one else self.K, self.V[0] if one else self.V, path, count,
                           nxt, out, **args)
        torch.cuda.synchronize()

    def check(self, n_nodes=None, parent=None, lengths=None):
        path, count, nxt, out = (t.cpu().numpy() for t in self.out)
        whole, pos = self.before
        K, V = (torch.as_strided(whole[j], self.K.shape, self.K.stride()) for j in range(2))
        for b in range(self.B):
            L = int(self.resp_len[b]) if lengths is None else int(lengths[b])
            n = int((self.n_nodes if n_nodes is None else n_nodes)[b])
            want, drawn = ort.accept_walk((self.parent if parent is None else parent)[b], n, self.draft[b], self.sampled[b],
                                          self.cap - L)
            assert list(path[b]) == want + [-1] * (self.N - len(want)), b
            assert count[b] == len(want) and nxt[b] == drawn and out[b] == L + len(want)
            if want:
                rows = torch.tensor([L + i for i in want], device="cuda")
                K[:, b, L:L + len(want)] = K[:, b, rows].clone()
                V[:, b, L:L + len(want)] = V[:, b, rows].clone()
                if pos is not None:
                    pos[b, L:L + len(want)] = pos[b, rows].clone()
        assert torch.equal(self.whole, whole)
        assert pos is None or torch.equal(self.pos, pos)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 5, 9, 17, 33, 64])
@pytest.mark.parametrize("shape", [(1, 1, 64), (3, 8, 128), (2, 5, 64), (1, 40, 128)], ids=lambda s: "%dx%dx%d" % s)
def test_walks_and_moves(ctx, dtype, N, shape):
    print("case:", dtype, N, shape, flush=True)
    for seed, in_place in ((N, False), (N + 50, True)):
        c = Case(dtype, 5, N, *shape, cap=N + 7, seed=seed, pad=16 if shape[0] > 1 else 0)
        c.call(ctx, in_place)
        c.check()


def test_long_chains_move_in_order(ctx):
    """every second node of a chain of brothers: each row moves onto one that another move reads"""
    c = Case("bf16", 4, 64, 2, 2, 64, cap=70, seed=3)
    c.parent = np.tile(np.array([-1] + [max(0, (i - 1) // 2 * 2) for i in range(1, 64)], np.int32), (4, 1))
    c.draft[:] = np.arange(64)
    c.sampled[:, ::2] = np.minimum(np.arange(0, 64, 2) + 2, 63)
    c.n_nodes[:] = [64, 63, 30, 1]
    c.call(ctx)
    c.check()
    assert list(c.out[1].cpu().numpy()) == [33, 32, 15, 1]     # 0, 2, ..., 62 and the leaf 63


def test_defaults_and_tables_out_of_contract(ctx):
    c = Case("bf16", 3, 8, 2, 2, 64, cap=20, seed=4, chain=True, resp=[0, 0, 0], agree=1.0)
    c.call(ctx, parent=None, n_nodes=None, resp_len=None, pos_resp=None)
    c.before = (c.before[0], None)
    c.pos = None
    c.check(n_nodes=[8, 8, 8])
    c = Case("f32", 3, 8, 2, 2, 64, cap=20, seed=5, chain=True, resp=[1, 2, 3], agree=1.0)
    c.call(ctx, parent=None, resp_len_add=4)
    c.check(lengths=c.resp_len + 4)
    # parents that do not come before are none, counts are clamped, nothing was sampled where it is negative
    c = Case("bf16", 4, 6, 1, 2, 64, cap=30, seed=6, resp=[1, 5, 9, 2])
    bad = np.array([[5, 0, 1, 2, 3, 4], [-1, 1, 0, 7, -9, 2], [-1, 0, 1, 2, 3, 4], [-1, 0, 1, 2, 3, 4]], np.int32)
    good = np.array([[-1, 0, 1, 2, 3, 4], [-1, -1, 0, -1, -1, 2], [-1, 0, 1, 2, 3, 4], [-1, 0, 1, 2, 3, 4]], np.int32)
    c.draft[:] = [9, 1, 2, 3, 4, 5]
    c.sampled[:] = [1, 2, 3, 4, 5, 6]
    c.draft[3, 1], c.sampled[3, 0] = -1, -1
    c.call(ctx, parent=dev(bad), n_nodes=dev(np.array([99, 6, -4, 1 << 30], np.int32)))
    c.check(n_nodes=[6, 6, 0, 6], parent=good)


@pytest.mark.parametrize("lengths", [[8, 9, 12, 14], [13, 15, 16, 40]])
def test_nodes_without_a_row_are_not_taken(ctx, lengths):
    c = Case("bf16", 4, 8, 2, 2, 64, cap=16, seed=7, resp=lengths, chain=True, agree=1.0)
    c.n_nodes[:] = 8
    c.call(ctx)
    c.check()


def test_graph_replays(ctx):
    """in place, so that each replay goes on from the one before"""
    c = Case("bf16", 3, 5, 2, 2, 64, cap=64, seed=8, resp=[0, 3, 6], agree=1.0)
    c.n_nodes[:] = 5
    lens, path, count, nxt = dev(c.resp_len), *c.out[:3]
    parent, n_nodes, draft, sampled = dev(c.parent), dev(c.n_nodes), dev(c.draft), dev(c.sampled)
    work = lambda: ctx.sp_tree_accept(draft, sampled, c.K, c.V, path, count, nxt, lens, parent=parent, n_nodes=n_nodes, resp_len=lens,
                                      pos_resp=c.pos)
    main = torch.cuda.current_stream().cuda_stream
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.sp_set_stream(torch.cuda.current_stream().cuda_stream)
        work()
    ctx.sp_set_stream(main)
    for rep in range(4):
        c.resp_len = lens.cpu().numpy()
        c.before = c.whole.clone(), c.pos.clone()
        g.replay()
        torch.cuda.synchronize()
        c.out[3] = lens
        c.check()
        _ = (c.K.float() * 2).sum()


def test_refusals(ctx):
    c = Case("bf16", 2, 4, 2, 2, 64, cap=8, seed=9)
    lens = dev(c.resp_len)
    path, count, nxt, out = c.out

    def status(draft=dev(c.draft), K=c.K, V=c.V, path=path, out=out, **kw):
        args = dict(parent=dev(c.parent), resp_len=lens)
        args.update(kw)
        with pytest.raises((B.SpError, ValueError)) as e:
            ctx.sp_tree_accept(draft, dev(c.sampled) if draft.shape[1] == 4 else draft, K, V, path, count, nxt, out, **args)
        return getattr(e.value, "status", None)

    many = torch.zeros((2, 65), dtype=torch.int32, device="cuda")
    assert status(draft=many, path=many.clone(), parent=None) == -3
    odd = torch.zeros((2, 2, 8, 2, 96), dtype=torch.bfloat16, device="cuda")
    assert status(K=odd, V=odd.clone()) == -3
    assert status(resp_len_add=-1) == -1
    both = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert status(resp_len=both[:2], out=both[1:]) == -1     # overlap
    assert status(K=c.K.float()) is None and status(V=c.V[:1]) is None and status(K=c.K.transpose(2, 3), V=c.V.transpose(2, 3)) is None
    assert status(K=c.K[:, ::2], V=c.V[:, ::2]) is None and status(n_nodes=lens[:1]) is None and status(path=path[:1]) is None
    near = torch.as_strided(c.whole[0], (2, 2, 8, 2, 64), (1024, 1024, 128, 64, 1))
    assert status(K=near, V=near) == -1                      # layers closer than a block
    torch.cuda.synchronize()
    assert all((t == -7).all() for t in c.out) and torch.equal(c.whole, c.before[0])
