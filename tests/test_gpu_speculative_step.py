"""A whole step of speculative decoding (speculate.TreeStep) over several layers: against the definitions, and recorded into a HIP
graph that is replayed with other trees, lengths and random numbers in the same tensors."""
import numpy as np
import pytest
import torch

from oracle import ref_numpy
from oracle import speculation as S
from paper_2511_21862_amd import binding as B
from paper_2511_21862_amd import workloads as W
from paper_2511_21862_amd.speculate import TreeStep

from gpu_util import say
from test_gpu_speculation import BF16, batch, bf16, bits, context, dev, trees

pytestmark = pytest.mark.gpu

HEADS, LAYERS, V, MAX_PATH = (8, 2, 128), 3, 997, 6


class Inputs:
    """A step's inputs on the host: trees of up to 12 nodes on up to 90 tokens, rows of every layer, probabilities."""

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.nodes, self.ctx = rng.integers(1, 13, 5), rng.integers(0, 91, 5).astype(np.int32)
        self.nodes[-1] += 50 - self.nodes.sum()          # 50 rows, so that a graph's sizes stay
        self.b = batch(HEADS, self.nodes.tolist(), self.ctx.tolist(), seed=600, spare=40 - sum(-(-(self.nodes + self.ctx) // 16)), max_blocks_per_seq=9)
        self.table = self.b.block_tables
        self.parents, self.qsl = trees(self.nodes, rng), self.b.query_start_loc
        std = lambda *s: W.f32_to_bf16_bits(rng.standard_normal(s, dtype=np.float32))
        self.qkv = std(LAYERS, 50, 12, 128)
        self.k, self.v = std(LAYERS, 40, 2, 16, 16, 8), std(LAYERS, 40, 2, 128, 16)
        z = rng.standard_normal((50, V)) * 3
        self.target = (np.exp(z) / np.exp(z).sum(-1, keepdims=True)).astype(np.float32)
        up = np.repeat(self.qsl[:-1], self.nodes) + np.maximum(self.parents, 0)
        self.tokens = np.argsort(-z[up], axis=1)[np.arange(50), rng.integers(0, 2, 50)].astype(np.int32)
        self.u, self.final = rng.random(50).astype(np.float32), rng.random(5).astype(np.float32)


class OnGpu:
    def __init__(self, x):
        self.parents, self.qsl, self.ctx, self.table, self.tokens, self.u, self.final, self.target = (
            dev(a) for a in (x.parents, x.qsl, x.ctx, x.table, x.tokens, x.u, x.final, x.target))
        self.qkv, self.k, self.v = bf16(x.qkv), bf16(x.k), bf16(x.v)
        self.out = torch.zeros((LAYERS, 50, 8, 128), dtype=torch.bfloat16, device="cuda")

    def take(self, o):
        for name, t in self.__dict__.items():
            t.copy_(getattr(o, name))

    def run(self, step):
        step.begin(self.parents, self.qsl, self.ctx, self.table)
        for i in range(LAYERS):
            q, k, v = self.qkv[i].split([8, 2, 2], dim=1)
            self.out[i].copy_(step.layer(q, k, v, self.k[i], self.v[i]))
        return step.finish(self.target, self.tokens, self.u, self.final, list(self.k), list(self.v))


FREQ = B.ooco_rope_frequencies("wavelength", 64, base=500000.0, scale=8.0, original_positions=8192, low=1.0, high=4.0)["frequencies"]


def check(x, g, counts, tokens):
    wide = ref_numpy.widen_bf16
    masks, pos = S.tree_masks(x.parents, x.qsl, x.ctx, 1)
    seq = np.repeat(np.arange(5), x.nodes)
    slot = x.ctx[seq] + np.arange(50) - x.qsl[seq]
    want_counts, path, want_tokens = S.verify_drafts(x.target.astype(np.float64), None, x.tokens, x.parents, x.u, x.final, x.qsl, MAX_PATH)
    assert (counts == want_counts).all() and (tokens == want_tokens).all()
    assert (g.ctx.cpu().numpy() == x.ctx + want_counts).all()
    out, k_gpu, v_gpu = bits(g.out), bits(g.k), bits(g.v)
    for i in range(LAYERS):
        rows = wide(x.qkv[i])
        # rotated q and k are rounded to bf16; k as the GPU has it (checked below), q by the same rounding
        q = W.bf16_bits_to_f32(W.f32_to_bf16_bits(S.rotate(rows[:, :8], pos, FREQ, False)[0].astype(np.float32))).astype(np.float64)
        k_new = S.rotate(rows[:, 8:10], pos, FREQ, False)
        k, v = wide(x.k[i]), wide(x.v[i])
        blk = x.table[seq, slot // 16]
        k[blk, :, :, slot % 16] = W.bf16_bits_to_f32(W.f32_to_bf16_bits(k_new[0].astype(np.float32))).reshape(50, 2, 16, 8)
        v[blk, :, :, slot % 16] = rows[:, 10:]
        tok = lambda pool, s, n: np.stack([pool[x.table[s, j // 16], ..., j % 16, :].reshape(2, 128) if pool.ndim == 5
                                           else pool[x.table[s, j // 16], :, :, j % 16] for j in range(n)])
        kv = [(tok(k, s, x.ctx[s] + x.nodes[s]), tok(v, s, x.ctx[s] + x.nodes[s])) for s in range(5)]
        want, size = S.attn_tree(q, [a for a, _ in kv], [a for _, a in kv], x.qsl, x.ctx, masks)
        # a q or k that the GPU rounds the other way (ties, sines a little off) moves a score by at most one step of its value: 2^-7 of
        # |q||k| / sqrt(hd), summed with random signs; 2^-5 of the spread of the values that a row sees covers it
        err = np.abs(wide(out[i]) - want)
        assert (err <= BF16 * np.abs(want) + (BF16 + 2.0 ** -5) * size).all() and np.sqrt((err ** 2).sum() / (want ** 2).sum()) <= 1e-2
        S.kv_compact(k, v, x.table, x.ctx, path, want_counts)
        err = np.abs(wide(k_gpu[i]) - k)
        assert (err <= 2 * BF16 * np.abs(k) + 2.0 ** -15).all() and (err > 0).mean() < 1e-3
        assert (wide(v_gpu[i]) == v).all()


def test_step():
    x = Inputs(0)
    say(f"case: speculative step, nodes={x.nodes.tolist()} ctx={x.ctx.tolist()}")
    g = OnGpu(x)
    with context(x.b) as c:
        c.rope_set(FREQ)
        step = TreeStep(c, rows=64, seqs=8, Hq=8, head_dim=128, max_path=MAX_PATH)
        counts, tokens = g.run(step)
        torch.cuda.synchronize()
        check(x, g, counts.cpu().numpy(), tokens.cpu().numpy())
        with pytest.raises(ValueError):
            step.begin(torch.zeros(65, dtype=torch.int32, device="cuda"), g.qsl, g.ctx, g.table)


def test_step_in_a_graph():
    inputs = [Inputs(i) for i in range(1, 5)]
    say("case: speculative step, captured and replayed")
    with context(inputs[0].b) as c:
        c.rope_set(FREQ)
        step = TreeStep(c, rows=50, seqs=5, Hq=8, head_dim=128, max_path=MAX_PATH)
        g = OnGpu(inputs[0])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            g.run(step)
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                counts, tokens = g.run(step)
        for x in inputs + inputs[:1]:
            fresh = OnGpu(x)
            g.take(fresh)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = counts.cpu().numpy().copy(), tokens.cpu().numpy().copy()
            check(x, g, *got)
            with torch.cuda.stream(side):        # the program's own eager step between the replays, to the same bits
                again = [t.cpu().numpy() for t in fresh.run(step)]
            side.synchronize()
            assert (again[0] == got[0]).all() and (again[1] == got[1]).all()
            assert (bits(fresh.out) == bits(g.out)).all() and (bits(fresh.k) == bits(g.k)).all() and (bits(fresh.v) == bits(g.v)).all()


def test_both_ways_of_marshalling_give_the_same(monkeypatch):
    x = Inputs(7)
    say("case: speculative step, native and general marshalling")
    results = []
    for native in (True, False):
        if native:
            assert B._native is not None
        else:
            for name in ("_masks_fast", "_rope_fast", "_tree_fast", "_verify_fast", "_compact_fast"):
                monkeypatch.setattr(B, name, B._not_native)
        g = OnGpu(x)
        with context(x.b) as c:
            c.rope_set(FREQ)
            counts, tokens = g.run(TreeStep(c, rows=50, seqs=5, Hq=8, head_dim=128, max_path=MAX_PATH))
            torch.cuda.synchronize()
            results.append([counts.cpu().numpy(), tokens.cpu().numpy(), bits(g.out), bits(g.k), bits(g.v)])
            with pytest.raises(B.OocoError) as e:          # the same refusals, too
                c.verify_drafts(g.target, g.tokens, g.u, g.final, g.qsl, counts, tokens[:, 1:].contiguous(), tokens, draft_probs=g.target,
                                parents=g.parents)
            assert e.value.status == B.OOCO_EINVAL and "chains" in e.value.message
    for a, b in zip(*results):
        assert (a == b).all()


def test_a_step_without_rows_leaves_the_lengths():
    say("case: step without rows")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    with B.Context(8, 2, 64, 16, 4, 2) as c:
        c.rope_set(B.ooco_rope_frequencies("plain", 64)["frequencies"])
        k, v = (torch.zeros((4, 2) + s, dtype=torch.bfloat16, device="cuda") for s in ((8, 16, 8), (64, 16)))
        step, lens = TreeStep(c, 16, 4, 8, 64), i32([5, 0, 17])
        step.begin(i32([]), i32([0, 0, 0, 0]), lens, i32([[0, 1], [2, -1], [3, 0]]))
        rows = lambda heads: torch.empty((0, heads, 64), dtype=torch.bfloat16, device="cuda")
        assert step.layer(rows(8), rows(2), rows(2), k, v).shape[0] == 0
        counts, _ = step.finish(torch.empty((0, 50), device="cuda"), i32([]), torch.empty(0, device="cuda"), torch.rand(3, device="cuda"), [k], [v])
        torch.cuda.synchronize()
    assert (counts == 0).all() and lens.tolist() == [5, 0, 17]
