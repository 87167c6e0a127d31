"""Operators of a speculative decoding step over the paged KV cache, and what each has to compute.

A step of speculation hands every sequence a tree of drafted tokens (its nodes; node 0 is the token that the last step
ended with) and runs the target model over all nodes at once:

  op "masks"    ooco_tree_masks: which nodes each node sees, from the nodes' parents, and the nodes' positions
  op "rope"     ooco_rope_append: rotary positions of q and k, the rotated k and the v into their paged slots
  op "attn"     ooco_attn_tree: the nodes' attention over the cached tokens and the nodes that each sees
  op "verify"   ooco_verify_drafts: which nodes the target's probabilities accept, and the token drawn after them
  op "compact"  ooco_kv_compact: the accepted nodes' K and V to the slots behind the cached tokens, all layers at once

Lengths belong to the case (its "lengths" number seeds them), values, trees and block tables to the seed of `prepare`.
Head layouts are those of the repository's configurations and tests.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

BS = 16          # tokens per KV block
HEADS = [(32, 8, 128), (64, 8, 128), (28, 4, 128), (32, 4, 64)]


# ------------------------------------------------------------------------------------------------- the cases
def _case(op, heads, lengths, seqs, nodes_lo, nodes_hi, ctx_lo, ctx_hi, chain=False, interleaved=False, rotary=0, given=True,
          vocab=0, draft=False, dtype="float32", layers=1, name=None):
    Hq, Hkv, hd = heads
    c = {"op": op, "Hq": Hq, "Hkv": Hkv, "hd": hd, "lengths": lengths, "seqs": seqs, "nodes_lo": nodes_lo, "nodes_hi": nodes_hi,
         "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "chain": chain, "interleaved": interleaved, "rotary": rotary or hd, "given": given,
         "vocab": vocab, "draft": draft, "dtype": dtype, "layers": layers}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one conversation with a small draft: everything is latency
        _case("masks", HEADS[0], 0, 1, 8, 8, 300, 300, name="masks-1"),
        # a full batch of wide trees
        _case("masks", HEADS[0], 1, 256, 20, 64, 100, 4000, name="masks-256"),
        # the nodes of eight sequences, positions by depth in the tree, half layout over the whole head
        _case("rope", HEADS[0], 2, 8, 9, 16, 500, 4000, name="rope-tree-8"),
        # prompts packed into one call, interleaved layout over half of the head, positions that follow the cache
        _case("rope", HEADS[0], 3, 5, 500, 1200, 0, 600, chain=True, interleaved=True, rotary=64, given=False, name="rope-prompts"),
        # one conversation, heads of 64: the shortest attention
        _case("attn", HEADS[3], 4, 1, 8, 8, 700, 700, name="attn-1"),
        # an ordinary batch: small trees on some thousand cached tokens
        _case("attn", HEADS[0], 5, 32, 5, 16, 512, 8192, name="attn-32"),
        # wide trees under many heads: as much matrix work as memory traffic
        _case("attn", HEADS[1], 6, 8, 64, 64, 12000, 16384, name="attn-wide"),
        # few sequences on long contexts, a group of seven heads
        _case("attn", HEADS[2], 7, 4, 20, 27, 60000, 131000, name="attn-long"),
        # sampled drafts: chains of five with the distributions that they were drawn from
        _case("verify", HEADS[0], 8, 64, 6, 6, 100, 4000, chain=True, vocab=128000, draft=True, name="verify-chain-64"),
        # trees of the draft's likeliest tokens, odd vocabulary, probabilities in bf16
        _case("verify", HEADS[0], 9, 4, 30, 60, 100, 4000, vocab=32003, dtype="bfloat16", name="verify-tree-4"),
        # accepted paths of one layer's cache
        _case("compact", HEADS[0], 10, 4, 16, 32, 100, 2000, name="compact-4"),
        # accepted paths of a whole model's cache
        _case("compact", HEADS[0], 11, 64, 16, 64, 100, 300, layers=32, name="compact-64x32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_KV_TOKENS = 450_000        # of 8 kv heads of 128 in one layer
MAX_PAIRS = 8_000_000          # (node, cached token) pairs of 64 query heads of 128
MAX_VALUES = 50_000_000        # probabilities


def draw(rng):
    """A case of the listed ranges: 1..256 sequences of 1..256 nodes on 0..131K cached tokens, prompts of 1..4096 rows."""
    while True:
        op = rng.choice(["masks", "rope", "rope", "attn", "attn", "attn", "verify", "verify", "compact"])
        heads = rng.choice(HEADS)
        hi = _log(rng, 1, 256 if op != "verify" else 64)
        ctx = _log(rng, 16, 131000 if op == "attn" else 4000)
        a = dict(heads=heads, lengths=rng.randrange(1 << 20), seqs=_log(rng, 1, 256), nodes_lo=max(1, hi // rng.choice([1, 2, 8])), nodes_hi=hi,
                 ctx_lo=rng.choice([0, ctx // 4, ctx]), ctx_hi=ctx, chain=rng.random() < 0.3)
        if op == "rope":
            a.update(interleaved=rng.random() < 0.5, rotary=rng.choice([16, 32, heads[2] // 2, heads[2]]), given=rng.random() < 0.5)
            if not a["given"]:
                rows = _log(rng, 1, 4096)
                a.update(nodes_lo=max(1, rows // 3), nodes_hi=rows)
        if op == "verify":
            a.update(vocab=_log(rng, 1000, 160000), dtype=rng.choice(["float32", "bfloat16"]), draft=a["chain"] and rng.random() < 0.7)
        if op == "compact":
            a.update(layers=_log(rng, 1, 64), ctx_lo=0, ctx_hi=rng.randint(0, 300))
        c = _case(op, **a)
        L = _lengths(c)
        rows, kv = int(L.nodes.sum()), int((L.ctx + L.nodes).sum())
        if op == "masks" and (c["chain"] or rows < 12) or op == "verify" and rows < 4:
            continue        # (nothing in them that another seed would change, or too little)
        heads_of = heads[0] * heads[2] / 8192
        if kv * c["layers"] * heads[1] * heads[2] > MAX_KV_TOKENS * 1024:
            continue
        if op == "attn" and int((L.nodes * L.ctx).sum()) * heads_of > MAX_PAIRS:
            continue
        if op == "rope" and rows > 4500:
            continue
        if op == "verify" and rows * c["vocab"] * (2 if c["draft"] else 1) > 2 * MAX_VALUES:
            continue
        return c


# ------------------------------------------------------------------------------------------------- lengths and work
def _lengths(c):
    """Nodes of each sequence and tokens cached before the step."""
    r = np.random.default_rng(c["lengths"])
    nodes = r.integers(c["nodes_lo"], c["nodes_hi"] + 1, size=c["seqs"])
    ctx = r.integers(c["ctx_lo"], c["ctx_hi"] + 1, size=c["seqs"])
    return SimpleNamespace(nodes=nodes, ctx=ctx, qsl=np.concatenate([[0], np.cumsum(nodes)]))


def _words(c):
    return (c["nodes_hi"] + 63) // 64


def _moved(c):
    """Accepted nodes of each sequence of a "compact" case."""
    L = _lengths(c)
    return np.minimum(np.random.default_rng(c["lengths"] + 1).integers(0, 9, size=c["seqs"]), (L.nodes - 1) // 2)


def work(c):
    L = _lengths(c)
    rows, kv, row = int(L.nodes.sum()), int((L.ctx + L.nodes).sum()), c["Hkv"] * c["hd"] * 2
    if c["op"] == "masks":
        return {"bytes": rows * (8 + 8 * _words(c)) + 8 * c["seqs"], "flops": rows}
    if c["op"] == "rope":
        both = c["Hq"] * c["hd"] * 2 + row
        return {"bytes": 2 * rows * (both + row), "flops": 3 * rows * (c["Hq"] + c["Hkv"]) * c["rotary"]}
    if c["op"] == "attn":
        return {"bytes": 2 * kv * row + 4 * rows * c["Hq"] * c["hd"] + 8 * rows * _words(c),
                "flops": 4 * c["Hq"] * c["hd"] * int((L.nodes * (L.ctx + 1)).sum())}
    if c["op"] == "verify":
        size = 4 if c["dtype"] == "float32" else 2
        return {"bytes": c["seqs"] * c["vocab"] * size * (2 if c["draft"] else 1) + 12 * rows, "flops": c["seqs"] * c["vocab"]}
    return {"bytes": max(1, 4 * int(_moved(c).sum()) * row * c["layers"]) + 8 * c["seqs"], "flops": 0}


# ------------------------------------------------------------------------------------------------- inputs
def _parents(c, L, rng):
    """Random trees: the parent of a node is any node before it; chains: the one before it.  The root has -1."""
    i = np.arange(int(L.nodes.max()))
    p = np.where(i > 0, i - 1, -1)[None] if c["chain"] else np.floor(rng.random((c["seqs"], len(i))) * i).astype(np.int64) - (i == 0)
    p = np.broadcast_to(p, (c["seqs"], len(i)))
    return p[i[None] < L.nodes[:, None]].astype(np.int32)


def _frequencies(c):
    """Base 500000, stretched by 8 in the manner of interpolated positions: the frequencies of the rotated pairs."""
    n = c["rotary"]
    return 500000.0 ** (-np.arange(0, n, 2, dtype=np.float64) / n) / 8.0


def _pools(s, c, blocks, g):
    k = torch.randn((c["layers"], blocks, c["Hkv"], c["hd"] // 8, BS, 8), generator=g, device="cuda", dtype=torch.bfloat16)
    v = torch.randn((c["layers"], blocks, c["Hkv"], c["hd"], BS), generator=g, device="cuda", dtype=torch.bfloat16)
    s.k, s.v = (k, v) if c["op"] == "compact" else (k[0], v[0])
    s.k_layers, s.v_layers = list(k), list(v)


def prepare(c, seed):
    rng = np.random.default_rng([seed, 17])
    g = torch.Generator(device="cuda").manual_seed(seed)
    L = _lengths(c)
    B, T, N = c["seqs"], int(L.nodes.sum()), int(L.nodes.max())
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    s = SimpleNamespace(**c, B=B, T=T, N=N, words=_words(c))
    s.qsl, s.ctx = dev(L.qsl.astype(np.int32)), dev(L.ctx.astype(np.int32))
    s.parents_host = _parents(c, L, rng)
    s.parents = dev(s.parents_host)
    if c["op"] in ("rope", "attn", "compact"):      # a block table over a shuffled pool
        need = -(-(L.ctx + L.nodes) // BS)
        s.blocks, s.per_seq = int(need.sum()) + 3, int(need.max())
        table = np.full((B, s.per_seq), -1, np.int32)
        table[np.arange(s.per_seq)[None] < need[:, None]] = rng.permutation(s.blocks)[:int(need.sum())]
        s.table = dev(table)
        _pools(s, c, s.blocks, g)
    if c["op"] == "rope":
        # q, k and v as a model's one projection leaves them: side by side in a row
        qkv = torch.randn((T, c["Hq"] + 2 * c["Hkv"], c["hd"]), generator=g, device="cuda", dtype=torch.bfloat16)
        s.q, s.k_new, s.v_new = qkv.split([c["Hq"], c["Hkv"], c["Hkv"]], dim=1)
        s.freq_host = _frequencies(c)
        s.freq = dev(s.freq_host)
        depth = _ancestors_host(s.parents_host, L).sum(-1) - 1 if c["given"] else None
        rows = np.arange(N)[None] < L.nodes[:, None]
        s.positions = dev((L.ctx[:, None] + depth)[rows].astype(np.int32)) if c["given"] else None
        s.q_out = torch.empty((T, c["Hq"], c["hd"]), dtype=torch.bfloat16, device="cuda")
    if c["op"] == "attn":
        s.q = torch.randn((T, c["Hq"], c["hd"]), generator=g, device="cuda", dtype=torch.bfloat16)
        see = _ancestors_host(s.parents_host, L)
        pad = np.zeros((B, N, s.words * 64), bool)
        pad[:, :, :N] = see
        bits = np.packbits(pad.reshape(B, N, s.words, 64), axis=-1, bitorder="little").view(np.int64)[..., 0]
        s.masks = dev(bits[np.arange(N)[None] < L.nodes[:, None]])
        s.out = torch.empty_like(s.q)
    if c["op"] == "masks":
        s.masks = torch.empty((T, s.words), dtype=torch.int64, device="cuda")
        s.positions = torch.empty(T, dtype=torch.int32, device="cuda")
    if c["op"] == "verify":
        _prepare_verify(s, c, L, g)
    if c["op"] == "compact":
        # paths whose nodes are not also places of other accepted nodes, so that a pass leaves what the next one reads
        moved = _moved(c)
        path = np.full((B, 8), -1, np.int32)
        for b in range(B):
            m = int(moved[b])
            path[b, :m] = m + 1 + np.sort(rng.choice(int(L.nodes[b]) - 1 - m, size=m, replace=False)) if m else 0
        s.path, s.counts = dev(path), dev((moved + 1).astype(np.int32))
    return s


def _ancestors_host(parents, L):
    """bool [B][N][N]: node i sees node j (itself and its ancestors)."""
    B, N = len(L.nodes), int(L.nodes.max())
    see = np.zeros((B, N, N), bool)
    p = np.full((B, N), -1)
    p[np.arange(N)[None] < L.nodes[:, None]] = parents
    b = np.arange(B)
    for i in range(N):
        has = p[:, i] >= 0
        see[b[has], i] = see[b[has], p[has, i]]
        see[i < L.nodes, i, i] = True
    return see


def _prepare_verify(s, c, L, g):
    T, V = s.T, c["vocab"]
    dtype = getattr(torch, c["dtype"])
    z = torch.randn((T, V), generator=g, device="cuda").mul_(3.0 if c["draft"] else 5.0)
    first = torch.from_numpy(L.qsl[:-1]).cuda().repeat_interleave(torch.from_numpy(L.nodes).cuda())
    up = (first + s.parents.clamp(min=0)).long()                       # row of the parent
    s.target = z.softmax(-1).to(dtype)
    s.draft = None
    if c["draft"]:      # tokens drawn from a distribution near the target's
        q = z[up].add_(torch.randn((T, V), generator=g, device="cuda").mul_(0.6)).softmax(-1)
        s.draft = q.to(dtype)
        r = torch.rand((T, 1), generator=g, device="cuda", dtype=torch.float64)
        s.tokens = torch.searchsorted(q.cumsum(-1, dtype=torch.float64), r).clamp(max=V - 1)[:, 0].to(torch.int32)
    else:               # the likeliest tokens after the parent, one for each of its children
        rank = np.zeros(T, np.int64)
        for i in range(len(L.nodes)):
            p = s.parents_host[L.qsl[i]:L.qsl[i + 1]]
            order = np.argsort(p, kind="stable")
            start = np.searchsorted(p[order], p[order])
            rank[L.qsl[i] + order] = np.arange(len(p)) - start
        top = z.topk(int(rank.max()) + 1, dim=-1).indices
        s.tokens = top[up, torch.from_numpy(rank).cuda()].to(torch.int32)
    s.uniforms = torch.rand(T, generator=g, device="cuda")
    s.final = torch.rand(s.B, generator=g, device="cuda")
    s.max_path = s.N - 1
    s.counts = torch.empty(s.B, dtype=torch.int32, device="cuda")
    s.path = torch.empty((s.B, s.N - 1), dtype=torch.int32, device="cuda")
    s.out_tokens = torch.empty((s.B, s.N), dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------- the framework's operators
_contexts = {}


def _context(s):
    """The program's handle for a layer geometry, made once and kept."""
    from paper_2511_21862_amd import binding

    blocks, per_seq = getattr(s, "blocks", 1), getattr(s, "per_seq", 1)
    key = (s.op, s.Hq, s.Hkv, s.hd, blocks, per_seq, s.rotary, s.interleaved)
    if key not in _contexts:
        ctx = _contexts[key] = binding.Context(s.Hq, s.Hkv, s.hd, BS, blocks, per_seq)
        if s.op == "rope":
            ctx.rope_set(s.freq_host, interleaved=s.interleaved)
    return _contexts[key]


def run(s):
    if not own:
        return _PLAIN[s.op](s)
    ctx = _context(s)
    if s.op == "masks":
        ctx.tree_masks(s.parents, s.qsl, s.ctx, s.masks, s.positions)
        return {"masks": s.masks, "positions": s.positions}
    if s.op == "rope":
        ctx.rope_append(s.q, s.k_new, s.v_new, s.q_out, s.k, s.v, s.table, s.qsl, s.ctx, positions=s.positions)
        return {"q": s.q_out, "k": s.k, "v": s.v}
    if s.op == "attn":
        ctx.attn_tree(s.q, s.k, s.v, s.table, s.qsl, s.ctx, s.masks, s.out)
        return s.out
    if s.op == "verify":
        ctx.verify_drafts(s.target, s.tokens, s.uniforms, s.final, s.qsl, s.counts, s.path, s.out_tokens,
                          draft_probs=s.draft, parents=None if s.chain else s.parents)
        return {"counts": s.counts, "path": s.path, "tokens": s.out_tokens}
    ctx.kv_compact(s.k_layers, s.v_layers, s.table, s.ctx, s.path, s.counts)
    return {"k": s.k, "v": s.v}


# ------------------------------------------------------------------------------------------------- plain forms
def _padded(s):
    """Rows of every sequence side by side: indices [B][N], which of them are rows, and each row's (sequence, node)."""
    n = s.qsl[1:] - s.qsl[:-1]
    t = torch.arange(s.N, device="cuda", dtype=torch.int32)
    at = (s.qsl[:-1, None] + t).clamp(max=s.T - 1).long()
    row = torch.arange(s.T, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s.qsl, row, right=True) - 1
    return at, t[None] < n[:, None], seq, (row - s.qsl[seq]).long()


def _sees(s, at, is_row):
    """[B][N][N]: node i sees node j, by powers of the parents' matrix."""
    par = torch.where(is_row, s.parents[at], -1).long()
    see = torch.zeros((s.B, s.N, s.N + 1), device="cuda")
    see.scatter_(2, torch.where(par < 0, s.N, par)[..., None], 1.0)
    see = see[..., :-1] + torch.eye(s.N, device="cuda")
    for _ in range(max(1, (s.N - 1).bit_length())):
        see = torch.matmul(see, see).clamp(max=1.0)
    return see > 0.5


def _plain_masks(s):
    at, is_row, seq, node = _padded(s)
    see = _sees(s, at, is_row)
    bits = torch.zeros((s.B, s.N, s.words * 64), dtype=torch.int64, device="cuda")
    bits[..., :s.N] = see
    one = torch.ones(64, dtype=torch.int64, device="cuda") << torch.arange(64, device="cuda")
    words = (bits.view(s.B, s.N, s.words, 64) * one).sum(-1)
    depth = (see.sum(-1, dtype=torch.int32) - 1)
    s.masks.copy_(words[seq, node])
    s.positions.copy_(s.ctx[seq] + depth[seq, node])
    return {"masks": s.masks, "positions": s.positions}


def _plain_rope(s):
    row = torch.arange(s.T, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s.qsl, row, right=True) - 1
    slot = (s.ctx[seq] + row - s.qsl[seq]).long()
    pos = slot if s.positions is None else s.positions
    angle = pos.double()[:, None] * s.freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotate(x):
        x = x.float()
        y, n = x.clone(), s.rotary
        a, b = (slice(0, n, 2), slice(1, n, 2)) if s.interleaved else (slice(0, n // 2), slice(n // 2, n))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y.bfloat16()

    s.q_out.copy_(rotate(s.q))
    block = s.table[seq, slot // BS].long()
    s.k[block, :, :, slot % BS] = rotate(s.k_new).view(s.T, s.Hkv, s.hd // 8, 8)
    s.v[block, :, :, slot % BS] = s.v_new
    return {"q": s.q_out, "k": s.k, "v": s.v}


def _plain_attn(s):
    at, is_row, seq, node = _padded(s)
    n, tokens, g = (s.qsl[1:] - s.qsl[:-1])[:, None, None], s.per_seq * BS, s.Hq // s.Hkv
    table = s.table.clamp(min=0).long()
    k = s.k[table].permute(0, 2, 3, 5, 1, 4).reshape(s.B, s.Hkv, s.hd, tokens).float()
    v = s.v[table].permute(0, 2, 1, 4, 3).reshape(s.B, s.Hkv, tokens, s.hd).float()
    q = s.q[at].view(s.B, s.N, s.Hkv, g, s.hd).permute(0, 2, 1, 3, 4).reshape(s.B, s.Hkv, s.N * g, s.hd).float()
    scores = torch.matmul(q, k).mul_(s.hd ** -0.5).view(s.B, s.Hkv, s.N, g, tokens)
    j = torch.arange(tokens, device="cuda")[None, None] - s.ctx[:, None, None]          # node that a token is
    word = s.masks[at].gather(2, (j.clamp(0, s.words * 64 - 1) >> 6).expand(s.B, s.N, tokens).long())
    sees = (j < 0) | ((j < n) & ((word >> (j.clamp(min=0) & 63)) & 1).bool())
    scores.masked_fill_(~sees[:, None, :, None], -math.inf)
    weights = (scores - scores.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = weights.sum(-1, keepdim=True)
    o = torch.matmul(weights.view(s.B, s.Hkv, s.N * g, tokens), v) / total.clamp(min=1e-30).view(s.B, s.Hkv, s.N * g, 1)
    o = o.view(s.B, s.Hkv, s.N, g, s.hd).permute(0, 2, 1, 3, 4).reshape(s.B, s.N, s.Hq, s.hd)
    s.out.copy_(o[seq, node])
    return s.out


def _plain_verify(s):
    at, is_row, seq, node = _padded(s)
    par = torch.where(is_row, s.parents[at], -1).long()
    up = at.gather(1, par.clamp(min=0))                                            # row of the parent
    tok = torch.where(is_row, s.tokens[at], -1).long()
    drafted = is_row & (par >= 0)
    p = s.target[up, tok.clamp(min=0)].double()
    q = s.draft[at, tok.clamp(min=0)].double() if s.draft is not None else torch.ones_like(p)
    i = torch.arange(s.N, device="cuda")
    sibling = (par[:, :, None] == par[:, None]) & drafted[:, :, None] & drafted[:, None] & (i[:, None] > i)     # [c][earlier j]
    again = (sibling & (tok[:, :, None] == tok[:, None])).any(-1)                  # a token that a sibling has had already
    p = p.masked_fill(again, 0.0)
    rest = 1.0 - torch.matmul(sibling.double(), p[..., None])[..., 0]
    accept = drafted & (s.uniforms[at].double() * q * rest < p)
    chosen = accept & ~(sibling & accept[:, None]).any(-1)
    chosen[:, 0] = True
    reached = is_row & ~(_sees(s, at, is_row) & ~chosen[:, None]).any(-1)          # all nodes up to the root are chosen
    taken = reached.sum(-1) - 1
    order = torch.where(reached, i, s.N).sort(-1).values                           # the nodes of the path, root first
    last = order.gather(1, taken[:, None])
    step = torch.arange(s.N, device="cuda")[None]
    s.path.copy_(torch.where(step[:, 1:] <= taken[:, None], order[:, 1:], -1))
    s.counts.copy_(taken + 1)
    # the token after the path: from what the rejected children leave of the last node's distribution
    row = at.gather(1, last)[:, 0]
    full = s.target[row].double()
    refused = drafted & (par == last)
    rest = full.clone()
    if s.draft is not None:
        child = torch.where(refused, i, 0).amax(-1)
        there = refused.any(-1, keepdim=True)
        rest -= torch.where(there, s.draft[at[torch.arange(s.B, device="cuda"), child]].double(), 0.0)
        rest.clamp_(min=0.0)
    else:
        rest = torch.cat([rest, rest[:, :1]], 1).scatter_(1, torch.where(refused, tok, s.vocab), 0.0)[:, :-1]
    rest = torch.where(rest.sum(-1, keepdim=True) > 0, rest, full)
    sums = rest.cumsum(-1)
    drawn = torch.searchsorted(sums, s.final.double()[:, None] * sums[:, -1:], right=True).clamp(max=s.vocab - 1)
    path_tok = tok.gather(1, torch.cat([order[:, 1:], order[:, :1]], 1).clamp(max=s.N - 1))
    s.out_tokens.copy_(torch.where(step < taken[:, None], path_tok, torch.where(step == taken[:, None], drawn, -1)))
    return {"counts": s.counts, "path": s.path, "tokens": s.out_tokens}


def _plain_compact(s):
    d = torch.arange(s.path.shape[1], device="cuda")
    moves = d[None] < s.counts[:, None] - 1
    src = s.ctx[:, None] + torch.where(moves, s.path, 0)        # (the others move the root onto itself)
    dst = s.ctx[:, None] + torch.where(moves, d + 1, 0)
    b = torch.arange(s.B, device="cuda")[:, None]
    sb, db = s.table[b, src // BS].long(), s.table[b, dst // BS].long()
    ss, ds = (src % BS).long(), (dst % BS).long()
    s.k[:, db, :, :, ds] = s.k[:, sb, :, :, ss]
    s.v[:, db, :, :, ds] = s.v[:, sb, :, :, ss]
    return {"k": s.k, "v": s.v}


_PLAIN = {"masks": _plain_masks, "rope": _plain_rope, "attn": _plain_attn, "verify": _plain_verify, "compact": _plain_compact}


# ------------------------------------------------------------------------------------------------- definitions in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    L = _lengths(c)
    return {"masks": _exact_masks, "rope": _exact_rope, "attn": _exact_attn, "verify": _exact_verify, "compact": _exact_compact}[c["op"]](s, L)


def _paths(s, L, b):
    """For each node of sequence b the nodes from the root to it."""
    paths = []
    for p in s.parents_host[L.qsl[b]:L.qsl[b + 1]].tolist():
        paths.append((paths[p] if p >= 0 else []) + [len(paths)])
    return paths


def _exact_masks(s, L):
    masks, positions = np.zeros((s.T, s.words), np.uint64), np.zeros(s.T, np.int32)
    for b in range(s.B):
        for t, path in enumerate(_paths(s, L, b)):
            row = L.qsl[b] + t
            positions[row] = L.ctx[b] + len(path) - 1
            for j in path:
                masks[row, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return {"masks": masks.view(np.int64), "positions": positions}


def _exact_rope(s, L):
    seq = np.repeat(np.arange(s.B), L.nodes)
    slot = L.ctx[seq] + np.arange(s.T) - L.qsl[seq]
    pos = slot if s.positions is None else s.positions.cpu().numpy()
    turn = np.exp(1j * (pos[:, None] * s.freq_host))[:, None]
    half = s.rotary // 2

    def rotate(x):
        x = x.cpu().double().numpy().copy()
        part = x[..., :s.rotary]
        pairs = part.reshape(*part.shape[:-1], half, 2) if s.interleaved else np.stack([part[..., :half], part[..., half:]], -1)
        z = (pairs[..., 0] + 1j * pairs[..., 1]) * turn
        both = np.stack([z.real, z.imag], -1)
        x[..., :s.rotary] = both.reshape(part.shape) if s.interleaved else np.concatenate([both[..., 0], both[..., 1]], -1)
        return x

    k, v, table = s.k.cpu().double().numpy(), s.v.cpu().double().numpy(), s.table.cpu().numpy()
    block = table[seq, slot // BS]
    k[block, :, :, slot % BS] = rotate(s.k_new).reshape(s.T, s.Hkv, s.hd // 8, 8)
    v[block, :, :, slot % BS] = s.v_new.cpu().double().numpy()
    return {"q": rotate(s.q), "k": k, "v": v}


def _exact_attn(s, L):
    out = torch.zeros((s.T, s.Hq, s.hd), dtype=torch.float64, device="cuda")
    group = s.Hq // s.Hkv
    for b in range(s.B):
        lo, hi, n = int(L.qsl[b]), int(L.qsl[b + 1]), int(L.ctx[b] + L.nodes[b])
        ids = s.table[b, :-(-n // BS)].long()
        allowed = torch.zeros((hi - lo, n), dtype=torch.bool)
        allowed[:, :int(L.ctx[b])] = True
        for t, path in enumerate(_paths(s, L, b)):
            allowed[t, [int(L.ctx[b]) + j for j in path]] = True
        allowed = allowed.cuda()
        for h in range(s.Hkv):
            k = s.k[ids, h].double().permute(0, 2, 1, 3).reshape(-1, s.hd)[:n]       # [token][dim]
            v = s.v[ids, h].double().transpose(1, 2).reshape(-1, s.hd)[:n]
            for r in range(group):
                x = (s.q[lo:hi, h * group + r].double() @ k.T.contiguous()) / math.sqrt(s.hd)
                out[lo:hi, h * group + r] = x.masked_fill(~allowed, -math.inf).softmax(-1) @ v
    return out


def _exact_verify(s, L):
    target, draft = s.target.cpu(), None if s.draft is None else s.draft.cpu()
    tokens, u, final = s.tokens.cpu().tolist(), s.uniforms.cpu().tolist(), s.final.cpu().tolist()
    counts, path, out = np.zeros(s.B, np.int32), np.full((s.B, s.N - 1), -1, np.int32), np.full((s.B, s.N), -1, np.int32)
    for b in range(s.B):
        lo = int(L.qsl[b])
        parents = s.parents_host[lo:L.qsl[b + 1]].tolist()
        at, taken, tried = 0, [], []
        while True:
            p = target[lo + at].double().numpy().copy()
            tried, left, step = [], 1.0, None
            for child in [i for i, up in enumerate(parents) if up == at]:
                x = tokens[lo + child]
                w = 0.0 if x in tried else float(p[x])
                if u[lo + child] * (1.0 if draft is None else float(draft[lo + child, x])) * left < w:
                    step = child
                    break
                tried.append(x)
                left -= w
                refused = child
            if step is None:
                break
            taken.append(step)
            at = step
        rest = p.copy()
        if tried and draft is not None:
            rest = np.maximum(p - draft[lo + refused].double().numpy(), 0.0)
        elif tried:
            rest[tried] = 0.0
        sums = np.cumsum(rest if rest.sum() > 0 else p)
        counts[b] = len(taken) + 1
        path[b, :len(taken)] = taken
        out[b, :len(taken) + 1] = [tokens[lo + i] for i in taken] + [min(int((sums <= final[b] * sums[-1]).sum()), s.vocab - 1)]
    return {"counts": counts, "path": path, "tokens": out}


def _exact_compact(s, L):
    k, v = s.k.double(), s.v.double()
    old_k, old_v, table, path, counts = s.k.double(), s.v.double(), s.table.cpu().numpy(), s.path.cpu().numpy(), s.counts.cpu().numpy()
    for b in range(s.B):
        for d in range(int(counts[b]) - 1):
            src, dst = int(L.ctx[b]) + int(path[b, d]), int(L.ctx[b]) + d + 1
            k[:, table[b, dst // BS], :, :, dst % BS] = old_k[:, table[b, src // BS], :, :, src % BS]
            v[:, table[b, dst // BS], :, :, dst % BS] = old_v[:, table[b, src // BS], :, :, src % BS]
    return {"k": k, "v": v}
