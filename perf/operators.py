"""Several tokens a step: the operators of a generation loop that drafts a tree of tokens and keeps what the model agrees with.

Kinds of case:
  tree    `sp_tree_decode`, one layer's attention of a tree of drafted tokens per prompt over the joined cache
          [preamble; kept paths; response] and the tokens' own ancestors, with their K/V appended to the response cache
  sample  `sp_sample`, a token for every row of logits (temperature, min-p, top-k, top-p, one given random number a row)
  accept  `sp_tree_accept`, the walk down the tree along the sampled tokens, and the accepted tokens' rows of all layers'
          response caches moved to where the next step expects them

Shapes are those of `sp_synth.WORKLOADS` and of `perf/cases.py`, and sizes around them.  Everything that is shape (document and
response lengths, trees, how far a walk gets) follows from the case alone; everything that is value follows from the seed.

`own` false: `run` computes the operators with elementary torch operations; true: by the library's entry points.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_TREE = {"kind": "tree", "dtype": "bf16", "prompts": 1, "hq": 32, "hkv": 32, "d": 128, "preamble": 64, "paths": 20, "doc_lo": 128,
         "doc_hi": 128, "query": 24, "k": 2, "resp_max": 255, "nodes": 16, "ragged": False, "shape": "random", "bias": False,
         "kv_layout": "token"}
_SAMPLE = {"kind": "sample", "dtype": "bf16", "rows": 1, "vocab": 50432, "logit_std": 3.0, "filters": "none", "rows_per_set": 1}
_ACCEPT = {"kind": "accept", "dtype": "bf16", "prompts": 1, "layers": 32, "hkv": 32, "d": 128, "capacity": 280, "resp_max": 255,
           "nodes": 16, "ragged": False, "shape": "random", "bias": False}


def _case(base, name=None, **kw):
    c = dict(base)
    c.update(kw)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # One user, five drafted tokens, the shape of a 7B model's layer: an interactive service, where latency counts.
        _case(_TREE, "tree_one_prompt", nodes=5, doc_lo=64, doc_hi=220, resp_max=60),
        # The benchmark's decode batch in the middle of its responses, trees of 16 tokens.
        _case(_TREE, "tree_mha_batch", prompts=64),
        # Grouped query heads, four kept paths, the widest trees there are: 256 query rows to a KV head.
        _case(_TREE, "tree_gqa_wide", prompts=16, hkv=8, preamble=96, doc_lo=160, doc_hi=160, k=4, nodes=64, resp_max=120),
        # Two long responses of a model with few KV heads: little to share out but the length.
        _case(_TREE, "tree_gqa_long", prompts=2, hkv=4, d=64, nodes=33, ragged=True, resp_max=12000, kv_layout="head"),
        # The fp32 precision path, with positions that act as a distance penalty, ragged trees.
        _case(_TREE, "tree_f32_bias", dtype="f32", prompts=6, hkv=8, preamble=96, doc_lo=64, doc_hi=220, k=4, nodes=12,
              ragged=True, resp_max=120, bias=True),
        # The next token of one user, nucleus sampling.
        _case(_SAMPLE, "sample_one_row", filters="top_p"),
        # A batch of users, each with settings of their own, the large vocabulary.
        _case(_SAMPLE, "sample_mixed_batch", rows=64, vocab=128256, filters="mixed"),
        # Every node of the 64 trees of the batch above, drawn from the model's own distribution.
        _case(_SAMPLE, "sample_tree_rows", rows=1024, rows_per_set=16),
        # An fp32 LM head with an odd vocabulary, the best 50 and of them the nucleus.
        _case(_SAMPLE, "sample_f32_top_k", dtype="f32", rows=96, vocab=50257, filters="top_k_p"),
        # One user's tree over the caches of 32 layers.
        _case(_ACCEPT, "accept_one_prompt", nodes=5, shape="wide", capacity=64, resp_max=50),
        # The batch, grouped heads.
        _case(_ACCEPT, "accept_gqa_batch", prompts=64, hkv=8),
        # fp32 caches with positions, ragged trees, some of them empty.
        _case(_ACCEPT, "accept_f32_ragged", dtype="f32", prompts=16, layers=8, nodes=24, ragged=True, bias=True),
    ]


# Most that a drawn case may cost (`work`), so that none costs more than the largest listed one of its kind.
_MOST_BYTES = {"tree": 6.0e8, "sample": 1.0e8, "accept": 2.0e8}
_MOST_FLOPS = {"bf16": 1.6e10, "f32": 1.0e9}


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["tree", "tree", "tree", "sample", "sample", "accept"])
        f32 = rng.random() < 0.25
        hq, hkv, d = rng.choice([(32, 32, 128), (32, 32, 128), (32, 8, 128), (32, 8, 128), (16, 16, 64), (32, 4, 64),
                                 (24, 24, 128), (12, 6, 128), (28, 4, 128)])
        nodes = log_int(1, 64)
        more = dict(dtype="f32" if f32 else "bf16", nodes=nodes, ragged=rng.random() < 0.5, bias=rng.random() < 0.3,
                    shape=rng.choice(["random", "wide", "chain"]))
        if kind == "tree":
            lo = log_int(24, 192)
            paths = log_int(4, 40)
            c = _case(_TREE, prompts=log_int(1, 64), hq=hq, hkv=hkv, d=d, preamble=log_int(12, 128), paths=paths, doc_lo=lo,
                      doc_hi=rng.choice([lo, min(256, lo + log_int(8, 160))]), query=log_int(4, 40),
                      k=min(paths, rng.choice([1, 2, 4])), resp_max=log_int(4, 4000), kv_layout=rng.choice(["token", "token", "head"]),
                      **more)
        elif kind == "sample":
            c = _case(_SAMPLE, dtype=more["dtype"], rows=log_int(1, 1024),
                      vocab=rng.choice([512, 32000, 50257, 50432, 128256, log_int(300, 130000)]),
                      logit_std=rng.choice([0.7, 2.0, 3.0, 5.0]),
                      filters=rng.choice(["none", "top_k", "top_p", "top_k_p", "min_p", "mixed", "greedy"]),
                      rows_per_set=rng.choice([1, 1, 4, 16]))
        else:
            resp = log_int(4, 1000)
            c = _case(_ACCEPT, prompts=log_int(1, 64), layers=log_int(1, 32), hkv=hkv, d=d, resp_max=resp,
                      capacity=resp + nodes + rng.randint(0, 40), **more)
        w = work(c)
        if w["bytes"] <= _MOST_BYTES[kind] and (kind != "tree" or w["flops"] <= _MOST_FLOPS[c["dtype"]]) and _state_bytes(c) <= 4e9:
            return c


# ---- shapes ------------------------------------------------------------------------------------------------------

def _shape_rng(c, what):
    return random.Random("%s %s" % (what, sorted((k, v) for k, v in c.items() if k != "name")))


def _esz(dtype):
    return 2 if dtype == "bf16" else 4


def _torch_dtype(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _trees(c):
    """Parents [prompts][nodes] (-1: a root), the number of nodes that each prompt has, and the nodes that its walk will take."""
    rng = _shape_rng(c, "trees")
    parents, n_nodes, walks = [], [], []
    for _ in range(c["prompts"]):
        n = rng.randint(0, c["nodes"]) if c["ragged"] else c["nodes"]
        if c["kind"] == "tree" or not c["ragged"]:
            n = max(n, 1)
        if c["shape"] == "chain":
            p = [i - 1 for i in range(c["nodes"])]
        elif c["shape"] == "wide":                         # every node has up to three children, in the order of a heap
            p = [-1] + [(i - 1) // 3 for i in range(1, c["nodes"])]
        else:
            p = [-1] + [rng.randint(max(0, i - 6), i - 1) for i in range(1, c["nodes"])]
        walk = []
        if n:
            walk = [0]
            while True:
                children = [i for i in range(1, n) if p[i] == walk[-1]]
                if not children or rng.random() < 0.15:
                    break
                walk.append(rng.choice(children))
        parents.append(p)
        n_nodes.append(n)
        walks.append(walk)
    return parents, n_nodes, walks


class _Table:
    """Segment table of a case, preamble -> {document -> its query copy} per prompt, tokens in that order."""

    def __init__(self, c):
        rng = _shape_rng(c, "lengths")
        off, start, length, parent, path = [0], [], [], [], []
        self.shared, self.paths, self.path_off = [], [], [0]    # (first token, tokens)
        tok = 0
        for _ in range(c["prompts"]):
            first = len(start)
            start.append(tok); length.append(c["preamble"]); parent.append(-1); path.append(-1)
            self.shared.append((tok, c["preamble"]))
            tok += c["preamble"]
            for j in range(c["paths"]):
                n = rng.randint(c["doc_lo"], c["doc_hi"])
                start += [tok, tok + n]; length += [n, c["query"]]; parent += [first, len(start) - 2]; path += [j, j]
                self.paths.append((tok, n + c["query"]))
                tok += n + c["query"]
            off.append(len(start))
            self.path_off.append(self.path_off[-1] + c["paths"])
        i32 = lambda a: np.asarray(a, np.int32)
        self.n_tokens = tok
        self.args = (i32(off), i32(start), i32(length), i32(parent), i32(path))
        self.resp_len = [rng.randint(c["resp_max"] // 2, c["resp_max"]) for _ in range(c["prompts"])]

    def positions(self):
        """Every token at its index in [preamble; document; query] of its path."""
        pos = np.zeros(self.n_tokens, np.float32)
        for a, n in self.shared:
            pos[a:a + n] = np.arange(n)
        P = self.shared[0][1]
        for a, n in self.paths:
            pos[a:a + n] = P + np.arange(n)
        return pos


def _state_bytes(c):
    e = _esz(c["dtype"])
    if c["kind"] == "tree":
        t = _Table(c)
        return 2 * c["hkv"] * c["d"] * e * (t.n_tokens + c["prompts"] * (c["resp_max"] + c["nodes"]))
    if c["kind"] == "sample":
        return c["rows"] * (c["vocab"] + 8) * e
    return 2 * c["layers"] * c["prompts"] * c["capacity"] * c["hkv"] * c["d"] * e


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    c, e = case, _esz(case["dtype"])
    if c["kind"] == "tree":
        t, (_, n_nodes, _) = _Table(c), _trees(c)
        keys = nodes = pairs = 0
        for b, n in enumerate(n_nodes):                    # the kept paths are values: their mean length stands for them
            mine = t.paths[t.path_off[b]:t.path_off[b + 1]]
            seen = t.shared[b][1] + c["k"] * sum(p[1] for p in mine) / len(mine) + t.resp_len[b]
            keys += seen
            nodes += n
            pairs += n * (seen + 1)
        # cached K and V once; the nodes' q, o, k, v and the copies of k, v that the cache gets
        return {"bytes": int(c["d"] * e * (2 * c["hkv"] * keys + nodes * (2 * c["hq"] + 4 * c["hkv"]))),
                "flops": int(4 * c["d"] * c["hq"] * pairs)}
    if c["kind"] == "sample":
        return {"bytes": c["rows"] * (c["vocab"] * e + 12), "flops": 4 * c["rows"] * c["vocab"]}
    moved = sum(sum(1 for j, i in enumerate(w) if i != j) for w in _trees(c)[2])
    return {"bytes": 4 * moved * c["layers"] * c["hkv"] * c["d"] * e + 16 * c["prompts"] * c["nodes"], "flops": 0}


# ---- a user's program ----------------------------------------------------------------------------------------------

_ctx = None


def _context():
    """The program's one library context, on torch's current stream."""
    global _ctx
    if _ctx is None:
        from paper_2404_06910_amd import binding as B
        _ctx = B.Context(torch.cuda.current_device())
    return _ctx


class _State:
    pass


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = _State()
    s.case = c
    dt = _torch_dtype(c["dtype"])

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    def ints(a):
        return torch.from_numpy(np.asarray(a, np.int32)).cuda()

    if c["kind"] == "sample":
        rows, V = c["rows"], c["vocab"]
        per = 16 // _esz(c["dtype"])                       # rows start at 16-byte boundaries, as an LM head pads them
        full = torch.randn((rows, (V + per - 1) // per * per), generator=g, device="cuda", dtype=dt).mul_(c["logit_std"])
        s.logits = full[:, :V]
        s.u = torch.rand(rows, generator=g, device="cuda")
        sets = (rows + c["rows_per_set"] - 1) // c["rows_per_set"]
        T, K, P, M = (np.full(sets, v, t) for v, t in ((1.0, np.float32), (0, np.int32), (1.0, np.float32), (0.0, np.float32)))
        kind = [["greedy", "top_k", "top_p", "min_p", "top_k_p", "none"][i % 6] if c["filters"] == "mixed" else c["filters"]
                for i in range(sets)]
        for i, f in enumerate(kind):
            if f != "none":
                T[i] = 0.0 if f == "greedy" else rng.uniform(0.6, 1.2)
            if f in ("top_k", "top_k_p"):
                K[i] = rng.integers(1, 101) if c["filters"] == "mixed" else 50
            if f in ("top_p", "top_k_p"):
                P[i] = rng.uniform(0.8, 0.98)
            if f == "min_p":
                M[i] = rng.uniform(0.02, 0.2)
        s.temperature, s.top_k, s.top_p, s.min_p = (torch.from_numpy(a).cuda() for a in (T, K, P, M))
        s.token = torch.zeros(rows, dtype=torch.int32, device="cuda")
        s.logprob = torch.zeros(rows, device="cuda")
        return s

    B, N, d = c["prompts"], c["nodes"], c["d"]
    parents, n_nodes, walks = _trees(c)
    s.parent, s.n_nodes = ints(parents), ints(n_nodes)
    if c["kind"] == "accept":
        shape_rng = _shape_rng(c, "responses")
        s.resp_len = ints([shape_rng.randint(c["resp_max"] // 2, c["resp_max"]) for _ in range(B)])
        draft = rng.integers(0, 50432, (B, N)) * 2         # odd tokens are none that was drafted
        sampled = rng.integers(0, 50432, (B, N)) * 2 + 1
        for b, w in enumerate(walks):
            for i, nxt in zip(w, w[1:]):
                for j in range(nxt):                       # no earlier brother drafts the same
                    if parents[b][j] == i and draft[b, j] == draft[b, nxt]:
                        draft[b, j] += 1
                sampled[b, i] = draft[b, nxt]
        s.draft, s.sampled = ints(draft), ints(sampled)
        s.K, s.V = (normal(c["layers"], B, c["capacity"], c["hkv"], d) for _ in range(2))
        s.pos = torch.rand((B, c["capacity"]), generator=g, device="cuda") * 500 if c["bias"] else None
        s.path = torch.zeros((B, N), dtype=torch.int32, device="cuda")
        s.n_accepted, s.next_token, s.len_out = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
        return s

    t = _Table(c)
    H, Hkv = c["hq"], c["hkv"]
    s.scale = 1.0 / math.sqrt(d)
    s.cap = max(t.resp_len) + N

    def cache(n):
        # token-major [n, heads, d], or a per-head cache seen as such a tensor
        return normal(Hkv, n, d).transpose(0, 1) if c["kv_layout"] == "head" else normal(n, Hkv, d)

    s.K, s.V = cache(t.n_tokens), cache(t.n_tokens)
    s.Kr, s.Vr = normal(B, s.cap, Hkv, d), normal(B, s.cap, Hkv, d)
    s.q, s.k_new, s.v_new = normal(B, N, H, d), normal(B, N, Hkv, d), normal(B, N, Hkv, d)
    s.o = torch.zeros_like(s.q)
    s.resp_len = ints(t.resp_len)
    s.kept = ints(np.stack([rng.permutation(c["paths"])[:c["k"]] for _ in range(B)]))
    pos = slopes = s.slopes = s.tok_pos = s.pos_resp = s.new_pos = None
    if c["bias"]:
        pos, slopes = t.positions(), np.exp2(-np.linspace(1.0, 8.0, H)).astype(np.float32)
        first = float(pos.max()) + 1.0
        s.tok_pos, s.slopes = torch.from_numpy(pos).cuda(), torch.from_numpy(slopes).cuda()
        s.pos_resp = first + torch.arange(s.cap, device="cuda", dtype=torch.float32).repeat(B, 1)
        depth = np.zeros((B, N), np.float32)
        for b in range(B):
            for i in range(N):
                depth[b, i] = depth[b, parents[b][i]] + 1 if parents[b][i] >= 0 else 0
        s.new_pos = first + s.resp_len.float()[:, None] + torch.from_numpy(depth).cuda()
    # where each path's tokens are, as a program that gathers them by itself keeps it
    longest = max(n for _, n in t.paths)
    table = np.full((B, c["paths"], longest), -1, np.int64)
    for b in range(B):
        for j, (a, n) in enumerate(t.paths[t.path_off[b]:t.path_off[b + 1]]):
            table[b, j, :n] = np.arange(a, a + n)
    s.path_tokens = torch.from_numpy(table).cuda()
    s.shared_tokens = torch.from_numpy(np.stack([np.arange(a, a + n) for a, n in t.shared])).cuda()
    if own:
        from paper_2404_06910_amd import binding as Bd
        s.plan = Bd.Plan(_context(), *t.args, t.n_tokens, H, Hkv, d, Bd.SP_BF16 if c["dtype"] == "bf16" else Bd.SP_F32, tok_pos=pos,
                         alibi_slopes=slopes)
    return s


def run(s):
    c = s.case
    if own:
        ctx = _context()
        if c["kind"] == "sample":
            ctx.sp_sample(s.logits, s.u, s.token, logprob=s.logprob, temperature=s.temperature, top_k=s.top_k, top_p=s.top_p,
                          min_p=s.min_p, rows_per_set=c["rows_per_set"])
            return {"token": s.token, "logprob": s.logprob}
        if c["kind"] == "accept":
            ctx.sp_tree_accept(s.draft, s.sampled, s.K, s.V, s.path, s.n_accepted, s.next_token, s.len_out, parent=s.parent,
                               n_nodes=s.n_nodes, resp_len=s.resp_len, pos_resp=s.pos)
            return _accepted(s)
        ctx.sp_tree_decode(s.plan, s.kept, c["k"], s.K, s.V, s.Kr, s.Vr, s.cap, s.q, s.k_new, s.v_new, s.o, s.scale,
                           parent=s.parent, n_nodes=s.n_nodes, resp_len=s.resp_len, pos_resp=s.pos_resp, new_pos=s.new_pos)
        return _decoded(s)
    return {"sample": _plain_sample, "accept": _plain_accept, "tree": _plain_tree}[c["kind"]](s)


def _accepted(s):
    out = {"K": s.K, "V": s.V, "path": s.path, "n_accepted": s.n_accepted, "next_token": s.next_token, "resp_len": s.len_out}
    return out if s.pos is None else dict(out, pos=s.pos)


def _decoded(s):
    out = {"o": s.o, "K_resp": s.Kr, "V_resp": s.Vr}
    return out if s.pos_resp is None else dict(out, pos_resp=s.pos_resp)


# ---- the operators in elementary operations --------------------------------------------------------------------------

def _ancestors(parent):
    """[B, N, N]: 1 where node j is node i or an ancestor of it (parents come first, so 64 nodes are reached in 6 doublings)."""
    B, N = parent.shape
    node = torch.arange(N, device=parent.device)
    reach = (parent[:, :, None] == node).float() + torch.eye(N, device=parent.device)
    for _ in range(6):
        reach = (torch.bmm(reach, reach) > 0).float()
    return reach


def _plain_tree(s):
    B, N, H, d = s.q.shape
    Hkv, cap = s.Kr.shape[2], s.cap
    kept = s.kept.long()
    joined = torch.cat([s.shared_tokens, torch.gather(s.path_tokens, 1, kept[:, :, None].expand(-1, -1, s.path_tokens.shape[2])).flatten(1)], 1)
    at, n, length = joined.clamp(min=0), s.n_nodes[:, None], s.resp_len[:, None]
    node, row = torch.arange(N, device=at.device), torch.arange(cap, device=at.device)
    live = node < n                                                            # [B, N]

    def keys(packed, resp, new):                                               # [B, Hkv, keys, d]
        return torch.cat([packed[at].float(), resp.float(), new.float()], 1).transpose(1, 2).contiguous()

    K, V = keys(s.K, s.Kr, s.k_new), keys(s.V, s.Vr, s.v_new)
    seen = torch.cat([(joined >= 0)[:, None].expand(-1, N, -1), (row < length)[:, None].expand(-1, N, -1),
                      (_ancestors(s.parent) > 0) & live[:, None]], 2)          # [B, N, keys]
    q = s.q.float().view(B, N, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    score = torch.matmul(q, K.transpose(2, 3).contiguous()).view(B, Hkv, H // Hkv, N, -1) * s.scale
    if s.slopes is not None:
        pos = torch.cat([s.tok_pos[at], s.pos_resp, s.new_pos], 1)
        score = score - s.slopes.view(1, Hkv, -1, 1, 1) * (s.new_pos[:, :, None] - pos[:, None])[:, None, None]
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, -1, p.shape[-1]), V).view(B, Hkv, H // Hkv, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, H, d)
    s.o.copy_(torch.where(live[:, :, None, None], o.to(s.o.dtype), s.o))
    # the nodes' K and V (and positions) to rows [length, length + n) of the response cache
    mine = row - length
    new_row, mine = (mine >= 0) & (mine < n), mine.clamp(0, N - 1).long()
    for cache, new in ((s.Kr, s.k_new), (s.Vr, s.v_new)) + (((s.pos_resp, s.new_pos),) if s.pos_resp is not None else ()):
        shape = (B, cap) + (1,) * (cache.dim() - 2)
        cache.copy_(torch.where(new_row.view(shape), torch.gather(new, 1, mine.view(shape).expand_as(cache)), cache))
    return _decoded(s)


def _plain_sample(s):
    rows, V = s.logits.shape
    each = torch.arange(rows, device=s.u.device) // s.case["rows_per_set"]
    T, k, top_p, min_p = s.temperature.double()[each], s.top_k[each], s.top_p.double()[each], s.min_p.double()[each]
    x, order = torch.sort(s.logits.double(), dim=1, descending=True, stable=True)
    T = torch.where(T > 0, T, 1.0)[:, None]
    w = torch.exp((x - x[:, :1]) / T)
    rank = torch.arange(V, device=x.device)
    greedy = s.temperature[each] <= 0
    limit = torch.where(k > 0, k, V)
    kept = (w >= min_p[:, None]) & (rank < torch.where(greedy, 1, limit)[:, None])
    w = w * kept
    before = torch.cumsum(w, 1) - w
    total = before[:, -1:] + w[:, -1:]
    kept &= (before < top_p[:, None] * total) | (top_p >= 1)[:, None] | (rank == 0)
    w = w * kept
    run_mass = torch.cumsum(w, 1)
    at = (run_mass <= s.u.double()[:, None] * run_mass[:, -1:]).sum(1, keepdim=True)
    at = torch.minimum(at, kept.sum(1, keepdim=True) - 1)
    s.token.copy_(torch.gather(order, 1, at)[:, 0])
    s.logprob.copy_(((torch.gather(x, 1, at) - x[:, :1]) / T - torch.log(run_mass[:, -1:]))[:, 0])
    return {"token": s.token, "logprob": s.logprob}


def _plain_accept(s):
    B, N = s.draft.shape
    node = torch.arange(N, device=s.draft.device)
    up = s.parent.clamp(min=0).long()
    same = (s.draft == torch.gather(s.sampled, 1, up)) & (s.parent >= 0) & (node < s.n_nodes[:, None])
    # of several brothers that draft the same token the first counts
    earlier = same[:, None] & (s.parent[:, None] == s.parent[:, :, None]) & (node[None, :] < node[:, None])
    good = same & ~earlier.any(2) | (node == 0)
    reach = _ancestors(s.parent)
    taken = (torch.bmm(reach, (~good).float()[:, :, None])[:, :, 0] == 0) & (reach[:, :, 0] > 0) & (s.n_nodes[:, None] > 0)
    count = taken.sum(1, keepdim=True)
    path = torch.sort(torch.where(taken, node, N), 1)[0]
    path = torch.where(node < count, path, -1)
    last = torch.gather(path, 1, (count - 1).clamp(min=0)).clamp(min=0)
    s.path.copy_(path)
    s.n_accepted.copy_(count[:, 0])
    s.next_token.copy_(torch.where(count > 0, torch.gather(s.sampled, 1, last), -1)[:, 0])
    s.len_out.copy_(s.resp_len + s.n_accepted)
    to = s.resp_len[:, None].long() + node                                     # a node that is not taken stays
    come = torch.where(path >= 0, s.resp_len[:, None] + path, to)
    b = torch.arange(B, device=to.device)[:, None]
    s.K[:, b, to] = s.K[:, b, come]
    s.V[:, b, to] = s.V[:, b, come]
    if s.pos is not None:
        s.pos[b, to] = s.pos[b, come]
    return _accepted(s)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"sample": _exact_sample, "accept": _exact_accept, "tree": _exact_tree}[case["kind"]](s)


def _exact_tree(s):
    """Prompt by prompt, node by node, over the list of keys that the node sees."""
    B, N, H, d = s.q.shape
    G = H // s.Kr.shape[2]
    parent, n_nodes, length, kept = (a.tolist() for a in (s.parent, s.n_nodes, s.resp_len, s.kept))
    out = torch.zeros((B, N, H, d), dtype=torch.float64, device="cuda")
    Kr, Vr = s.Kr.double(), s.Vr.double()
    pos_resp = None if s.pos_resp is None else s.pos_resp.double()
    for b in range(B):
        toks = torch.cat([s.shared_tokens[b]] + [s.path_tokens[b, j] for j in kept[b]])
        toks = toks[toks >= 0]
        L = length[b]
        K = torch.cat([s.K[toks].double(), Kr[b, :L], s.k_new[b].double()])
        V = torch.cat([s.V[toks].double(), Vr[b, :L], s.v_new[b].double()])
        old = len(toks) + L
        for i in range(n_nodes[b]):
            chain, j = [], i
            while j >= 0:
                chain.append(old + j)
                j = parent[b][j]
            which = torch.tensor(list(range(old)) + chain[::-1], device="cuda")
            k = K[which].repeat_interleave(G, 1)
            z = (k * s.q[b, i].double()).sum(2) * s.scale
            if s.slopes is not None:
                where = torch.cat([s.tok_pos[toks].double(), pos_resp[b, :L], s.new_pos[b].double()])[which]
                z = z - (s.new_pos[b, i].double() - where)[:, None] * s.slopes.double()
            a = torch.softmax(z, 0)
            out[b, i] = (a[:, :, None] * V[which].repeat_interleave(G, 1)).sum(0)
    for b in range(B):
        L, n = length[b], n_nodes[b]
        Kr[b, L:L + n], Vr[b, L:L + n] = s.k_new[b, :n].double(), s.v_new[b, :n].double()
        if pos_resp is not None:
            pos_resp[b, L:L + n] = s.new_pos[b, :n].double()
    found = {"o": out, "K_resp": Kr, "V_resp": Vr}
    return found if pos_resp is None else dict(found, pos_resp=pos_resp)


def _exact_sample(s):
    """Row by row on the host."""
    X, u = s.logits.double().cpu().numpy(), s.u.double().cpu().numpy()
    T, k, P, M = (a.double().cpu().numpy() for a in (s.temperature, s.top_k, s.top_p, s.min_p))
    token, logprob = np.zeros(len(X), np.int32), np.zeros(len(X))
    for r, x in enumerate(X):
        i = r // s.case["rows_per_set"]
        if T[i] <= 0:
            token[r], logprob[r] = int(np.argmax(x)), 0.0
            continue
        order = np.argsort(-x, kind="stable")
        z = (x[order] - x[order[0]]) / T[i]
        w = np.exp(z)
        w = w[: int((w >= M[i]).sum())]
        w = w[: int(k[i])] if k[i] > 0 else w
        if P[i] < 1:
            reached = np.searchsorted(np.cumsum(w), P[i] * w.sum())      # the first whose running mass is enough
            w = w[: max(1, min(len(w), reached + 1))]
        mass = np.cumsum(w)
        j = min(int(np.searchsorted(mass, u[r] * mass[-1], side="right")), len(w) - 1)
        token[r], logprob[r] = order[j], z[j] - math.log(mass[-1])
    return {"token": token, "logprob": logprob}


def _exact_accept(s):
    """Prompt by prompt, one step of the walk after the other."""
    draft, sampled, parent, n_nodes, length = (a.tolist() for a in (s.draft, s.sampled, s.parent, s.n_nodes, s.resp_len))
    K, V = s.K.double(), s.V.double()
    pos = None if s.pos is None else s.pos.double()
    path, next_token = np.full(s.path.shape, -1, np.int32), np.full(len(draft), -1, np.int32)
    count, new_len = np.zeros(len(draft), np.int32), np.asarray(length, np.int32)
    for b, n in enumerate(n_nodes):
        at = 0 if n else -1
        while at >= 0:
            path[b, count[b]] = at
            count[b] += 1
            next_token[b] = sampled[b][at]
            at = next((i for i in range(n) if parent[b][i] == at and draft[b][i] == sampled[b][at]), -1)
        rows = torch.tensor([length[b] + int(i) for i in path[b, :count[b]]], dtype=torch.long, device="cuda")
        new_len[b] += count[b]
        for a in (K, V):
            a[:, b, length[b]:length[b] + len(rows)] = a[:, b, rows].clone()
        if pos is not None:
            pos[b, length[b]:length[b] + len(rows)] = pos[b, rows].clone()
    found = {"K": K, "V": V, "path": path, "n_accepted": count, "next_token": next_token, "resp_len": new_len}
    return found if pos is None else dict(found, pos=pos)
