"""The whole loop as a program runs it: prefill, saliency, pruning, then drafted trees -> sp_tree_decode per layer -> logits of every
node -> sp_sample -> sp_tree_accept.  A toy model of two layers generates the same tokens, and the same caches, as one token at a time."""
import math

import numpy as np
import pytest
import torch

import sp_synth
from paper_2404_06910_amd import binding as B

from gpu_util import make_plan

pytestmark = pytest.mark.gpu

H, HKV, D, VOCAB, LAYERS, CAP = 4, 2, 64, 96, 2, 48


class Toy:
    """q, k, v of a token: a table per layer, plus (from the second layer on) a mixture of the layer below's attention output."""

    def __init__(self, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.q, self.k, self.v = (r(LAYERS, VOCAB, n * D) for n in (H, HKV, HKV))
        self.mix = [r(H * D, n * D) / math.sqrt(H * D) for n in (H, HKV, HKV)]
        self.head = r(H * D, VOCAB) * 2
        self.scale = 1 / math.sqrt(D)

    def qkv(self, layer, tokens, below):
        out = []
        for table, mix, n in zip((self.q, self.k, self.v), self.mix, (H, HKV, HKV)):
            x = table[layer][tokens]
            if below is not None:
                x = x + torch.matmul(below.flatten(-2), mix)
            out.append(x.unflatten(-1, (n, D)).contiguous())
        return out


class Session:
    """What the cache holds after prefill and pruning, and the response so far."""

    def __init__(self, ctx, model, seed):
        rng = np.random.default_rng(seed)
        self.ctx, self.m = ctx, model
        lens = [[int(x) for x in rng.integers(3, 30, 5)] for _ in range(3)]
        self.st = st = sp_synth.forkjoin_segtable(7, lens, 4)
        self.B, self.k = 3, 2
        self.plan = make_plan(ctx, st, H, HKV, D, "f32")
        tokens = torch.from_numpy(rng.integers(0, VOCAB, st.n_tokens)).cuda()
        self.K, self.V, below = [], [], None
        for layer in range(LAYERS):
            q, k, v = model.qkv(layer, tokens, below)
            below = torch.zeros_like(q)
            ctx.sp_forkjoin_prefill(self.plan, q, k, v, below, model.scale)
            self.K.append(k)
            self.V.append(v)
        rows = np.concatenate([np.arange(st.seg_tok_start[s], st.seg_tok_start[s] + st.seg_tok_len[s]) for s in st.query_seg])
        logits = torch.matmul(below[torch.from_numpy(rows).cuda()].flatten(1), model.head)
        score = torch.zeros(st.n_slots, device="cuda")
        target = torch.from_numpy(rng.integers(0, VOCAB, len(rows)).astype(np.int32)).cuda()
        ctx.sp_path_saliency(logits, target, torch.from_numpy(np.repeat(np.arange(st.n_slots, dtype=np.int32), 4)).cuda(), st.n_slots, score)
        self.kept = torch.zeros((self.B, self.k), dtype=torch.int32, device="cuda")
        ctx.sp_prune_topk(score, self.plan.path_offsets_device(), self.B, 5, self.k, self.kept)
        self.Kr, self.Vr = (torch.zeros((LAYERS, self.B, CAP, HKV, D), device="cuda") for _ in range(2))
        self.len = torch.zeros(self.B, dtype=torch.int32, device="cuda")
        self.u = torch.rand((CAP + 1, self.B), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")

    def one_by_one(self, first, steps, temperature):
        cur, out = first, [first]
        for i in range(steps):
            below = None
            for layer in range(LAYERS):
                q, k, v = self.m.qkv(layer, cur.long(), below)
                below = torch.zeros_like(q)
                self.ctx.sp_pruned_decode(self.plan, self.kept, self.k, self.K[layer], self.V[layer], self.Kr[layer], self.Vr[layer], CAP,
                                          q, k, v, below, self.m.scale, resp_len=self.len)
            logits = torch.matmul(below.flatten(1), self.m.head)
            nxt = torch.zeros(self.B, dtype=torch.int32, device="cuda")
            self.ctx.sp_sample(logits, self.u[i], nxt, temperature=temperature)
            self.len += 1
            cur = nxt
            out.append(cur)
        return torch.stack(out, 1).cpu().numpy()

    def by_trees(self, first, steps, temperature, truth, rng):
        """Trees of up to 9 nodes: a path that follows the truth for a while, and wrong brothers.  u[i] goes with the i-th token."""
        N = 9
        done = [[int(t)] for t in first.cpu().numpy()]
        n_calls = 0
        while min(len(d) for d in done) <= steps:
            draft = rng.integers(0, VOCAB, (self.B, N)).astype(np.int32)
            parent = np.full((self.B, N), -1, np.int32)
            n_nodes = np.zeros(self.B, np.int32)
            for b in range(self.B):
                if len(done[b]) > steps:
                    continue                                   # finished: a prompt without nodes
                draft[b, 0] = done[b][-1]
                at, depth, n = 0, 0, int(rng.integers(1, N + 1))
                for i in range(1, n):
                    parent[b, i] = at if rng.random() < 0.8 else rng.integers(0, i)
                    if parent[b, i] == at and rng.random() < 0.8 and len(done[b]) + depth < len(truth[b]):
                        draft[b, i] = truth[b][len(done[b]) + depth]
                        at, depth = i, depth + 1
                n_nodes[b] = min(n, steps + 1 - len(done[b]))
            dev = lambda a: torch.from_numpy(a).cuda()
            d, p, n = dev(draft), dev(parent), dev(n_nodes)
            below = None
            for layer in range(LAYERS):
                q, k, v = self.m.qkv(layer, d.long(), below)
                below = torch.zeros_like(q)
                self.ctx.sp_tree_decode(self.plan, self.kept, self.k, self.K[layer], self.V[layer], self.Kr[layer], self.Vr[layer], CAP,
                                        q, k, v, below, self.m.scale, parent=p, n_nodes=n, resp_len=self.len)
            logits = torch.matmul(below.flatten(2), self.m.head).flatten(0, 1)
            depth = np.zeros((self.B, N), np.int64)
            for b in range(self.B):
                for i in range(1, N):
                    depth[b, i] = depth[b, parent[b, i]] + 1 if parent[b, i] >= 0 else 0
            place = np.minimum(depth + np.array([len(x) - 1 for x in done])[:, None], CAP)
            u = self.u[dev(place), torch.arange(self.B, device="cuda")[:, None]].flatten().contiguous()
            sampled = torch.zeros((self.B, N), dtype=torch.int32, device="cuda")
            self.ctx.sp_sample(logits, u, sampled, temperature=temperature, rows_per_set=N)
            path = torch.zeros_like(sampled)
            count, nxt = torch.zeros_like(self.len), torch.zeros_like(self.len)
            self.ctx.sp_tree_accept(d, sampled, self.Kr, self.Vr, path, count, nxt, self.len, parent=p, n_nodes=n, resp_len=self.len)
            path, count, nxt = path.cpu().numpy(), count.cpu().numpy(), nxt.cpu().numpy()
            for b in range(self.B):
                done[b] += [int(draft[b, i]) for i in path[b, 1:count[b]]] + ([int(nxt[b])] if count[b] else [])
            n_calls += 1
        return np.array([x[:steps + 1] for x in done]), n_calls


@pytest.mark.parametrize("temperature", [0.0, 0.8])
@pytest.mark.parametrize("seed", [1, 2])
def test_trees_generate_what_single_tokens_do(temperature, seed):
    ctx = B.Context(0)
    model = Toy(seed)
    steps = 24
    print("case:", temperature, seed, flush=True)
    rng = np.random.default_rng(seed)
    T = torch.full((3,), temperature, device="cuda")
    first = torch.tensor([3, 50, 77], dtype=torch.int32, device="cuda")
    a, b = Session(ctx, model, seed), Session(ctx, model, seed)
    assert torch.equal(a.kept, b.kept)
    truth = a.one_by_one(first, steps, T)
    got, calls = b.by_trees(first, steps, T, truth, rng)
    assert np.array_equal(got, truth)
    assert calls < steps                                       # several tokens a step
    assert list(b.len.cpu().numpy()) == [steps] * 3
    # K and V of the second layer carry the first one's attention, summed in another order: 64 products, ~100 keys, twice over,
    # values of a few units: 2^-24 * 4 * (64 + 100) * 2 * 8
    assert (a.Kr[:, :, :steps] - b.Kr[:, :, :steps]).abs().max() < 7e-4 and (a.Vr[:, :, :steps] - b.Vr[:, :, :steps]).abs().max() < 7e-4
    a.plan.close()
    b.plan.close()
    ctx.close()
