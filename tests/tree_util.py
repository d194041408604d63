"""What the tests of trees of drafted tokens share: trees, inputs, the call, the comparison with the 64-bit oracle."""
import math

import numpy as np
import torch

import sp_synth
from oracle import sp_oracle as orc
from oracle import sp_oracle_tree as ort

from gpu_util import TORCH_DT, dev, make_plan


def random_parents(rng, B, N):
    """[B, N], with several roots now and then"""
    out = np.full((B, N), -1, np.int32)
    for b in range(B):
        for i in range(1, N):
            out[b, i] = -1 if rng.random() < 0.05 else rng.integers(0, i)
    return out


class TreeCase:
    """A plan, a kept table, caches and a tree per prompt; arrays in fp32 as the device sees them."""

    def __init__(self, dtype, Hq, Hkv, d, N, B=2, paths=3, doc=(5, 40), query=4, preamble=11, k=2, resp=(0, 9), bias=False, seed=0,
                 packing="interleaved", room=3, n_nodes=None):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype, self.dims, self.N, self.B, self.k = rng, dtype, (Hq, Hkv, d), N, B, k
        lens = [[int(x) for x in rng.integers(doc[0], doc[1] + 1, paths)] for _ in range(B)]
        self.st = st = sp_synth.forkjoin_segtable(preamble, lens, query, packing)
        r = lambda *s: sp_synth.round_to_dtype(rng.standard_normal(s, dtype=np.float32), dtype)
        self.K, self.V = r(st.n_tokens, Hkv, d), r(st.n_tokens, Hkv, d)
        self.resp_len = rng.integers(resp[0], resp[1] + 1, B).astype(np.int32)
        self.cap = int(self.resp_len.max()) + N + room
        self.Kr, self.Vr = r(B, self.cap, Hkv, d), r(B, self.cap, Hkv, d)
        self.q, self.kn, self.vn = r(B, N, Hq, d), r(B, N, Hkv, d), r(B, N, Hkv, d)
        self.parent = random_parents(rng, B, N)
        self.n_nodes = np.asarray(n_nodes, np.int32) if n_nodes is not None else rng.integers(0, N + 1, B).astype(np.int32)
        self.kept = np.stack([rng.permutation(paths)[:k] for _ in range(B)]).astype(np.int32) if k else np.zeros((B, 0), np.int32)
        self.scale = 1 / math.sqrt(d)
        self.tok_pos = self.slopes = self.pos_resp = self.new_pos = None
        if bias:
            self.tok_pos, self.slopes = sp_synth.classical_positions(st), sp_synth.geometric_slopes(Hq)
            first = float(self.tok_pos.max()) + 1
            self.pos_resp = np.tile(first + np.arange(self.cap, dtype=np.float32), (B, 1))
            depth = np.array([[len(ort.lineage(p, i)) - 1 for i in range(N)] for p in self.parent], np.float32)
            self.new_pos = (first + self.resp_len[:, None] + depth).astype(np.float32)

    def plan(self, ctx):
        return make_plan(ctx, self.st, *self.dims, self.dtype, self.tok_pos, self.slopes)

    def upload(self):
        t = {n: dev(getattr(self, n), self.dtype) for n in ("K", "V", "Kr", "Vr", "q", "kn", "vn")}
        t["o"] = torch.full(self.q.shape, 7.0, dtype=TORCH_DT[self.dtype], device="cuda")
        for n in ("parent", "n_nodes", "kept", "resp_len", "pos_resp", "new_pos"):
            a = getattr(self, n)
            t[n] = None if a is None else dev(a)
        return t

    def call(self, ctx, plan, t, **kw):
        args = dict(parent=t["parent"], n_nodes=t["n_nodes"], resp_len=t["resp_len"], pos_resp=t["pos_resp"], new_pos=t["new_pos"])
        args.update(kw)
        ctx.sp_tree_decode(plan, t["kept"], self.k, t["K"], t["V"], t["Kr"], t["Vr"], self.cap, t["q"], t["kn"], t["vn"], t["o"],
                           self.scale, **args)

    def old_keys(self, b, length=None):
        """(K, V, positions) that every node of prompt b sees"""
        st = self.st
        idx = orc.joined_cache_index(st.prompt_seg_off, st.seg_tok_start, st.seg_tok_len, st.seg_path, b, self.kept[b])
        n = int(self.resp_len[b]) if length is None else length
        pos = None if self.tok_pos is None else np.concatenate([self.tok_pos[idx], self.pos_resp[b, :n]])
        return np.concatenate([self.K[idx], self.Kr[b, :n]]), np.concatenate([self.V[idx], self.Vr[b, :n]]), pos

    def check(self, t, n_nodes=None, parent=None, lengths=None, prompts=None):
        """o against the oracle; rows of nodes that are not there, and the response cache, bit for bit."""
        got = t["o"].float().cpu().numpy()
        nodes = self.n_nodes if n_nodes is None else n_nodes
        for b in range(self.B) if prompts is None else prompts:
            n = int(nodes[b])
            assert (got[b, n:] == 7).all()
            L = int(self.resp_len[b]) if lengths is None else int(lengths[b])
            Kr, Vr = self.Kr[b].copy(), self.Vr[b].copy()
            stored = max(0, min(n, self.cap - L))
            Kr[L:L + stored], Vr[L:L + stored] = self.kn[b, :stored], self.vn[b, :stored]
            assert np.array_equal(t["Kr"][b].float().cpu().numpy(), Kr) and np.array_equal(t["Vr"][b].float().cpu().numpy(), Vr)
            if self.pos_resp is not None:
                pos = self.pos_resp[b].copy()
                pos[L:L + stored] = self.new_pos[b, :stored]
                assert np.array_equal(t["pos_resp"][b].cpu().numpy(), pos)
            if n == 0:
                continue
            K, V, pos = self.old_keys(b, min(L, self.cap))
            up = (self.parent if parent is None else parent)[b]
            o, absum, big = ort.tree_attention(self.q[b, :n], self.kn[b, :n], self.vn[b, :n], K, V, up, self.scale, self.slopes,
                                               None if self.new_pos is None else self.new_pos[b], pos)
            # A score is off by at most (d + 8) roundings of `big` (products, their sum, the factor log2 e, the penalty), a
            # weight by twice that in relation, the sums over the keys by one rounding a key; bf16 rounds the weights and
            # the result once more each, by half a step.
            eps = 2.0 ** -24
            tol = absum * eps * (2 * (self.dims[2] + 8) * 1.45 * big[..., None] + len(K) + n + 16)
            if self.dtype == "bf16":
                tol = tol + 2.0 ** -8 * (absum + np.abs(o))
            off = np.abs(got[b, :n] - o)
            assert not np.isnan(got[b, :n]).any()
            assert (off <= tol).all(), "prompt %d: %.3g of the bound" % (b, (off / tol).max())
