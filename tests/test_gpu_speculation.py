"""GPU parity of the speculative decoding step's operators (through the C ABI) against their float64 definitions.

Tolerances.  A value that is rounded once to bf16 is off by at most 2^-8 of itself.  Rotation: each product and the sum are rounded to
fp32, and cosine and sine are off by at most 2^-17 together (the turn is held in fp32, half a step of 2^-24 of it being 2^-22 of the
angle; the hardware's own error is below 2^-18, 2^-22.9 as measured).  Attention: the weights are rounded to bf16 before they meet V (2^-8 of every
weight), the output once more; 2^-10 of sum(weight |v|) stands for everything held in fp32: scores of magnitude up to 30 in log2 units
with a few roundings of 2^-24 of sums of |q||k| each, exponentials and sums."""
import numpy as np
import pytest
import torch

from oracle import ref_numpy
from oracle import speculation as S
from paper_2511_21862_amd import binding as B
from paper_2511_21862_amd import workloads as W

from gpu_util import say

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8
HEADS = [(32, 8, 128), (64, 8, 128), (28, 4, 128), (32, 4, 64), (16, 1, 64), (3, 3, 128)]


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def context(b, **kw):
    return B.Context(b.Hq, b.Hkv, b.hd, b.BS, b.num_blocks, b.max_blocks_per_seq, **kw)


def batch(heads, nodes, ctx, seed, spare=5, **kw):
    Hq, Hkv, hd = heads
    need = sum((n + c + 15) // 16 for n, c in zip(nodes, ctx))
    return W.build_batch(Hq=Hq, Hkv=Hkv, hd=hd, q_lens=nodes, ctx_lens=ctx, num_blocks=need + spare, seed=seed, **kw)


def trees(nodes, rng, kind="random"):
    rows = []
    for n in nodes:
        i = np.arange(n)
        rows.append(i - 1 if kind == "chain" else np.where(i > 0, 0, -1) if kind == "star"
                    else np.where(i > 0, np.floor(rng.random(n) * i), -1))
    return np.concatenate(rows + [np.zeros(0)]).astype(np.int32)


def starts(nodes):
    return np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)


# ------------------------------------------------------------------------------------------------ masks
@pytest.mark.parametrize("words, nodes", [(1, [1]), (1, [0, 3, 64, 0, 2, 17]), (1, [70, 5]), (2, [65, 128, 1]), (3, [192, 130, 64]),
                                          (4, [256, 255, 193, 1, 0]), (4, [300, 2]), (1, [7] * 300)],
                         ids=lambda x: f"{len(x)}-seqs" if isinstance(x, list) else str(x))
@pytest.mark.parametrize("kind", ["random", "chain", "star"])
def test_masks(words, nodes, kind):
    rng = np.random.default_rng(words)
    ctx = rng.integers(0, 5000, len(nodes)).astype(np.int32)
    par, qsl = trees(nodes, rng, kind), starts(nodes)
    say(f"case: masks {words} {nodes[:6]} {kind}")
    want, pos = S.tree_masks(par, qsl, ctx, words)
    T = len(par)
    masks, positions = torch.full((T + 2, words), -7, dtype=torch.int64, device="cuda"), torch.full((T + 2,), -7, dtype=torch.int32, device="cuda")
    with B.Context(4, 1, 64, 16, 1, 1) as c:
        c.tree_masks(dev(par), dev(qsl), dev(ctx), masks, positions)
        only = torch.empty((T, words), dtype=torch.int64, device="cuda")
        c.tree_masks(dev(par), dev(qsl), dev(ctx), only)
        torch.cuda.synchronize()
    assert (masks[:T].cpu().numpy().view(np.uint64) == want).all() and (only == masks[:T]).all()
    assert (positions[:T].cpu().numpy() == pos).all()
    assert (masks[T:] == -7).all() and (positions[T:] == -7).all()       # rows behind the last sequence stay


def test_masks_of_parents_that_are_none():
    # later nodes, the node itself, far numbers and negative ones count as no parent
    par = np.array([-1, 1, 0, 5, 3, -9, 2 ** 31 - 1, 6, -2 ** 31], np.int32)
    say("case: masks of bad parents")
    want, pos = S.tree_masks(par, [0, 9], [11], 1)
    masks, positions = torch.empty((9, 1), dtype=torch.int64, device="cuda"), torch.empty(9, dtype=torch.int32, device="cuda")
    with B.Context(4, 1, 64, 16, 1, 1) as c:
        c.tree_masks(dev(par), dev(np.array([0, 9], np.int32)), dev(np.array([11], np.int32)), masks, positions)
        assert (masks.cpu().numpy().view(np.uint64) == want).all() and (positions.cpu().numpy() == pos).all()
        masks.fill_(5)      # rows that the arrays place outside the tensors are left alone
        c.tree_masks(dev(par), dev(np.array([3, 12], np.int32)), dev(np.array([11], np.int32)), masks, positions)
        c.tree_masks(dev(par), dev(np.array([4, 2], np.int32)), dev(np.array([11], np.int32)), masks, positions)
        torch.cuda.synchronize()
    assert (masks == 5).all()


# ------------------------------------------------------------------------------------------------ rotary positions and append
def check_rope(b, frequencies, interleaved, factor, positions, q, k_new, v_new, run):
    """run(ctx, device batch, table, qsl, ctx_lens, positions) -> q_out"""
    T = b.total_q
    seq = np.repeat(np.arange(b.num_seqs), b.q_lens)
    slot = b.ctx_lens[seq] + np.arange(T) - b.query_start_loc[seq]
    pos = slot if positions is None else positions
    d = W.to_device(b)
    with context(b) as c:
        c.rope_set(frequencies, interleaved=interleaved, factor=factor)
        q_out = run(c, d, dev(b.block_tables), dev(b.query_start_loc), dev(b.ctx_lens), None if positions is None else dev(positions))
        torch.cuda.synchronize()
    wide = ref_numpy.widen_bf16

    def close(got, x):
        want, size = S.rotate(wide(x), pos, frequencies, interleaved, factor)
        err = np.abs(wide(got) - want)
        assert (err <= BF16 * np.abs(want) + 2.0 ** -17 * size).all(), float((err - BF16 * np.abs(want)).max())
        rest = 2 * len(frequencies)
        assert (got[..., rest:] == x[..., rest:]).all()      # dims that are not rotated keep their bits

    close(bits(q_out), q)
    k, v = bits(d.k_cache), bits(d.v_cache)
    ok = slot // 16 < b.max_blocks_per_seq
    blk = b.block_tables[seq[ok], slot[ok] // 16]
    got = k[blk, :, :, slot[ok] % 16].reshape(-1, b.Hkv, b.hd)
    want, size = S.rotate(wide(k_new[ok]), pos[ok], frequencies, interleaved, factor)
    assert (np.abs(wide(got) - want) <= BF16 * np.abs(want) + 2.0 ** -17 * size).all()
    assert (v[blk, :, :, slot[ok] % 16] == v_new[ok]).all()
    k_rest, v_rest, k0, v0 = k.copy(), v.copy(), b.k_cache.copy(), b.v_cache.copy()
    for x in (k_rest, k0):
        x[blk, :, :, slot[ok] % 16] = 0
    for x in (v_rest, v0):
        x[blk, :, :, slot[ok] % 16] = 0
    assert (k_rest == k0).all() and (v_rest == v0).all()      # nothing else changed


def new_rows(b, seed):
    rng = np.random.default_rng(seed)
    return [W.f32_to_bf16_bits(rng.standard_normal((b.total_q, h, b.hd), dtype=np.float32)) for h in (b.Hq, b.Hkv, b.Hkv)]


ROWS = [([1], [0]), ([1, 1, 5, 0, 40], [36, 15, 16, 7, 3]), ([33, 1, 2], [0, 31, 47]), ([17, 100, 16, 2, 31], [15, 5, 16, 14, 1])]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [16, 32, 48, 0])
def test_rope_append(heads, interleaved, rotary):
    f = B.ooco_rope_frequencies("plain", rotary or heads[2], base=10000.0)["frequencies"]
    for i, (nodes, ctx) in enumerate(ROWS):
        b = batch(heads, nodes, ctx, seed=300 + i)
        say(f"case: rope {heads} interleaved={interleaved} rotary={rotary} rows={nodes}")
        q, k, v = new_rows(b, i)
        # (given: depths in a tree, far positions among them)
        given = None if i % 2 else np.random.default_rng(i).integers(0, 200000, b.total_q).astype(np.int32)

        def run(c, d, bt, qsl, cl, pos):
            out = torch.empty((b.total_q, b.Hq, b.hd), dtype=torch.bfloat16, device="cuda")
            c.rope_append(bf16(q), bf16(k), bf16(v), out, d.k_cache, d.v_cache, bt, qsl, cl, positions=pos)
            return out

        check_rope(b, f, interleaved, 1.0 if i % 2 else 1.25, given, q, k, v, run)


@pytest.mark.parametrize("place", ["one projection", "in place", "far apart"])
def test_rope_append_of_rows_inside_wider_tensors(place):
    b = batch(HEADS[2], [3, 20, 1], [14, 0, 63], seed=310)
    say(f"case: rope rows {place}")
    q, k, v = new_rows(b, 5)
    f = B.ooco_rope_frequencies("linear", 64, base=500000.0, scale=4.0)["frequencies"]

    def run(c, d, bt, qsl, cl, pos):
        T = b.total_q
        if place == "in place":
            out = bf16(q)
            c.rope_append(out, bf16(k), bf16(v), out, d.k_cache, d.v_cache, bt, qsl, cl)
            return out
        wide = torch.zeros((T, b.Hq + 2 * b.Hkv + (0 if place == "one projection" else 3), b.hd), dtype=torch.bfloat16, device="cuda")
        parts = wide[:, :b.Hq], wide[:, b.Hq:b.Hq + b.Hkv], wide[:, b.Hq + b.Hkv:b.Hq + 2 * b.Hkv]
        for part, x in zip(parts, (q, k, v)):
            part.copy_(bf16(x))
        out = torch.empty((T, b.Hq, b.hd), dtype=torch.bfloat16, device="cuda")
        c.rope_append(*parts, out, d.k_cache, d.v_cache, bt, qsl, cl)
        return out

    check_rope(b, f, False, 1.0, None, q, k, v, run)


def test_rope_append_far_positions_and_large_frequencies():
    # angles of 10^9 radians: the turns are reduced in 64 bits
    b = batch(HEADS[3], [6], [2], seed=311)
    say("case: rope far positions")
    q, k, v = new_rows(b, 6)
    pos = np.array([2 ** 30, 2 ** 31 - 1, 131071, 10 ** 9 + 7, 0, -5], np.int32)

    def run(c, d, bt, qsl, cl, p):
        out = torch.empty((b.total_q, b.Hq, b.hd), dtype=torch.bfloat16, device="cuda")
        c.rope_append(bf16(q), bf16(k), bf16(v), out, d.k_cache, d.v_cache, bt, qsl, cl, positions=p)
        return out

    check_rope(b, np.array([1.0, 0.5, 3.25, 1e-3, 0.0, 1e-6, 0.9, 2.0]), False, 1.0, pos, q, k, v, run)


def test_rope_append_of_rows_without_a_place():
    # a block id outside the pool, and rows past the block table: rotated, not appended
    b = batch(HEADS[3], [4, 4], [3, 20], seed=312)
    say("case: rope rows without a place")
    q, k, v = new_rows(b, 7)
    f = B.ooco_rope_frequencies("plain", 64)["frequencies"]
    table = b.block_tables.copy()
    table[1, 1] = 10 ** 6
    d = W.to_device(b)
    out = torch.full((8, b.Hq, b.hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    with context(b) as c:
        c.rope_set(f)
        cl = np.array([16 * b.max_blocks_per_seq - 2, 20], np.int32)       # two rows of the first sequence have a slot
        k0 = bits(d.k_cache).copy()
        c.rope_append(bf16(q), bf16(k), bf16(v), out, d.k_cache, d.v_cache, dev(table), dev(b.query_start_loc), dev(cl))
        torch.cuda.synchronize()
    want, size = S.rotate(ref_numpy.widen_bf16(q), np.concatenate([cl[0] + np.arange(4), 20 + np.arange(4)]), f, False)
    assert (np.abs(ref_numpy.widen_bf16(bits(out)) - want) <= BF16 * np.abs(want) + 2.0 ** -17 * size).all()
    changed = (bits(d.k_cache) != k0).any(axis=(1, 2, 4))
    blk = int(table[0, -1])
    assert blk < 0 and not changed.any() or changed.sum() == 2 and changed[blk, 14:].all()


# ------------------------------------------------------------------------------------------------ attention
def run_attn(b, masks, ctx=None, out=None, **kw):
    d = W.to_device(b)
    out = torch.full((b.total_q + 1, b.Hq, b.hd), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    words = masks.shape[1]
    with context(b, **kw) as c:
        B.ooco_attn_tree(c.h, d.q, d.k_cache, d.v_cache, dev(b.block_tables), dev(b.query_start_loc), dev(b.ctx_lens),
                         dev(masks.view(np.int64)), words, out, b.num_seqs, b.total_q)
        torch.cuda.synchronize()
    assert torch.isnan(out[b.total_q:]).all()        # the row behind the last sequence stays
    return bits(out[:b.total_q])


def check_attn(b, masks, got=None, scale=None, **kw):
    got = run_attn(b, masks, **kw) if got is None else got
    kv = [[ref_numpy.widen_bf16(x) for x in W.gather_logical(b, i)] for i in range(b.num_seqs)]
    want, size = S.attn_tree(ref_numpy.widen_bf16(b.q), [x[0] for x in kv], [x[1] for x in kv], b.query_start_loc, b.ctx_lens, masks, scale)
    err = np.abs(ref_numpy.widen_bf16(got) - want)
    worst = float((err - BF16 * np.abs(want) - (BF16 + 2.0 ** -10) * size).max()) if err.size else 0.0
    say(f"  rows {b.total_q}: max error {err.max() if err.size else 0:.3g}, beyond the bound by {worst:.3g}")
    assert np.isfinite(err).all() and worst <= 0


TREES = [([1], [0]), ([1], [1000]), ([8], [700]), ([5, 0, 16, 1, 33, 64], [100, 7, 0, 511, 31, 260]), ([3] * 9, [0, 1, 15, 16, 17, 127, 128, 129, 95]),
         ([64, 40], [3, 1500]), ([20, 2], [0, 2500])]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("kind", ["random", "chain"])
def test_attn_tree(heads, kind):
    for i, (nodes, ctx) in enumerate(TREES):
        b = batch(heads, nodes, ctx, seed=400 + i, poison=True)
        rng = np.random.default_rng(i)
        masks, _ = S.tree_masks(trees(nodes, rng, kind), b.query_start_loc, b.ctx_lens, 1)
        say(f"case: tree attention {heads} {kind} nodes={nodes} ctx={ctx}")
        check_attn(b, masks)


@pytest.mark.parametrize("words, nodes, ctx", [(2, [128, 70, 1], [40, 0, 333]), (3, [190], [1000]), (4, [256, 255, 100], [77, 16, 0]),
                                               (1, [100, 65], [50, 0]), (4, [10, 300], [9, 20])], ids=str)
@pytest.mark.parametrize("heads", [HEADS[0], HEADS[2], HEADS[3]], ids=str)
def test_attn_tree_of_many_nodes(heads, words, nodes, ctx):
    # masks of several words; nodes that the masks have no bits for see the cache and are seen by nobody
    b = batch(heads, nodes, ctx, seed=420, poison=True)
    masks, _ = S.tree_masks(trees(nodes, np.random.default_rng(1)), b.query_start_loc, b.ctx_lens, words)
    say(f"case: tree attention {heads} words={words} nodes={nodes}")
    check_attn(b, masks)


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[3]], ids=str)
def test_attn_tree_of_any_masks(heads):
    # masks that are no trees: later nodes, none at all, bits behind the last node; rows that see nothing are zero
    nodes, ctx = [30, 64, 5, 3, 90], [0, 11, 0, 40, 0]
    b = batch(heads, nodes, ctx, seed=430, poison=True)
    rng = np.random.default_rng(2)
    masks = rng.integers(0, 2 ** 63, (b.total_q, 2), dtype=np.uint64) * np.uint64(2) + rng.integers(0, 2, (b.total_q, 2), dtype=np.uint64)
    masks[3] = masks[94] = masks[98] = masks[100] = 0
    say(f"case: tree attention of any masks {heads}")
    got = run_attn(b, masks)
    check_attn(b, masks, got)
    assert (got[3] & 0x7FFF == 0).all() and (got[94] & 0x7FFF == 0).all() and (got[98] & 0x7FFF == 0).all()


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1], HEADS[3]], ids=str)
def test_attn_tree_long_contexts_are_cut_and_merged(heads):
    for nodes, ctx in (([7, 30], [9000, 130]), ([64], [6000]), ([1, 2, 3], [5000, 40, 7001])):
        b = batch(heads, nodes, ctx, seed=440)
        masks, _ = S.tree_masks(trees(nodes, np.random.default_rng(3)), b.query_start_loc, b.ctx_lens, 1)
        say(f"case: tree attention {heads} nodes={nodes} ctx={ctx}")
        first = run_attn(b, masks)
        check_attn(b, masks, first)
        assert (run_attn(b, masks) == first).all()                                   # the same bits again
        check_attn(b, masks, workspace_bytes=600 << 10)                              # a workspace of two runs


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[2], HEADS[3]], ids=str)
def test_attn_tree_of_wide_trees_and_large_tables(heads):
    # more than 128 columns a sequence and block tables of a capacity that calls for workgroups of eight waves: tiles of every width
    for nodes, ctx, words in (([64, 50, 64], [300, 1000, 17], 1), ([200, 130, 3, 0, 1, 70], [100, 0, 700, 5, 31, 64], 4), ([64], [9000], 1)):
        Hq, Hkv, hd = heads
        b = batch(heads, nodes, ctx, seed=435, poison=len(nodes) > 1, max_blocks_per_seq=-(-16 * 256 * 8 // (len(nodes) * Hkv)) + 1)
        masks, _ = S.tree_masks(trees(nodes, np.random.default_rng(3)), b.query_start_loc, b.ctx_lens, words)
        say(f"case: tree attention of wide trees {heads} nodes={nodes}")
        first = run_attn(b, masks)
        check_attn(b, masks, first)
        assert (run_attn(b, masks) == first).all()


@pytest.mark.parametrize("heads, seqs", [(HEADS[0], 66), (HEADS[3], 130), (HEADS[2], 130)], ids=str)
def test_attn_tree_of_whole_units(heads, seqs):
    # so many small trees that two workgroups to a compute unit find whole units, with a wide one among them
    rng = np.random.default_rng(7)
    nodes, ctx = rng.integers(0, 10, seqs).tolist(), rng.integers(0, 200, seqs).tolist()
    nodes[3], nodes[17], nodes[40] = 12, 64, 25
    b = batch(heads, nodes, ctx, seed=455, poison=True)
    masks, _ = S.tree_masks(trees(nodes, rng), b.query_start_loc, b.ctx_lens, 1)
    say(f"case: tree attention {heads} {seqs} sequences")
    first = run_attn(b, masks)
    check_attn(b, masks, first)
    assert (run_attn(b, masks) == first).all()


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[3], HEADS[4]], ids=str)
def test_attn_tree_of_trees_of_every_width(heads):
    # tiles of one, two and four times 32 columns in runs that cut them; and the same without the wide tree
    g = heads[0] // heads[1]
    for rows in ([10 * 4, 45 * 4, 5 * 4, 30 * 4], [10 * 4, 15 * 4, 5 * 4, 1]):
        nodes, ctx = [max(1, r // g) for r in rows], [2500, 500, 1900, 130]
        b = batch(heads, nodes, ctx, seed=456)
        masks, _ = S.tree_masks(trees(nodes, np.random.default_rng(8)), b.query_start_loc, b.ctx_lens, 1)
        say(f"case: tree attention {heads} nodes={nodes} ctx={ctx}")
        first = run_attn(b, masks)
        check_attn(b, masks, first)
        assert (run_attn(b, masks) == first).all()


def test_attn_tree_many_sequences():
    # more sequences than a workgroup looks at in one go
    rng = np.random.default_rng(4)
    nodes, ctx = rng.integers(0, 6, 700).tolist(), rng.integers(0, 90, 700).tolist()
    b = batch(HEADS[5], nodes, ctx, seed=450)
    masks, _ = S.tree_masks(trees(nodes, rng), b.query_start_loc, b.ctx_lens, 1)
    say("case: tree attention 700 sequences")
    check_attn(b, masks)


def test_attn_tree_scores_far_apart():
    # scores of some hundreds, rising over the keys: the running maximum moves often; a scale of one's own
    b = batch(HEADS[0], [9, 4], [800, 300], seed=460, value_std=4.0)
    masks, _ = S.tree_masks(trees([9, 4], np.random.default_rng(5)), b.query_start_loc, b.ctx_lens, 1)
    say("case: tree attention of large scores")
    check_attn(b, masks, scale=0.3, got=run_attn(b, masks, scale=0.3))


def test_attn_tree_nan_and_infinities():
    # K of a node that a row does not see may be anything; what a row sees of NaN or +inf reaches that row's heads alone
    heads, nodes, ctx = HEADS[0], [6], [200]
    b = batch(heads, nodes, ctx, seed=470)
    par = np.array([-1, 0, 0, 1, 2, 2], np.int32)
    masks, _ = S.tree_masks(par, b.query_start_loc, b.ctx_lens, 1)
    want = run_attn(b, masks)
    for value in (0x7FC0, 0x7F80, 0xFF80):
        blk, slot = int(b.block_tables[0, 202 // 16]), 202 % 16       # node 2: seen by nodes 2, 4 and 5
        bad = W.Batch(**{**b.__dict__, "k_cache": b.k_cache.copy()})
        bad.k_cache[blk, 3, :, slot, :] = value                       # kv head 3: query heads 12 .. 15
        say(f"case: tree attention, K of a node is {value:#x}")
        got = run_attn(bad, masks)
        reached = np.zeros_like(got, bool)
        reached[[2, 4, 5], 12:16] = True
        assert (got[~reached] == want[~reached]).all()
        assert np.isnan(ref_numpy.widen_bf16(got[reached])).all()      # (sums of both signs of infinity)


def test_attn_tree_lowest_scores():
    # a row whose every score is the lowest finite one, or -inf at some keys
    b = batch(HEADS[3], [3], [40], seed=480)
    b.q[:] = W.f32_to_bf16_bits(np.zeros(b.q.shape, np.float32))
    b.q[1, :, 0] = 0x7F00                                              # 2^127
    for j in range(43):
        blk, slot = int(b.block_tables[0, j // 16]), j % 16
        b.k_cache[blk, :, 0, slot, 0] = 0xC080 if j % 2 else 0x0000    # -4 (the product overflows to -inf) or 0
    masks, _ = S.tree_masks(np.array([-1, 0, 1], np.int32), b.query_start_loc, b.ctx_lens, 1)
    say("case: tree attention of lowest scores")
    kv = [[ref_numpy.widen_bf16(x) for x in W.gather_logical(b, 0)]]
    want, size = S.attn_tree(ref_numpy.widen_bf16(b.q), [kv[0][0]], [kv[0][1]], b.query_start_loc, b.ctx_lens, masks)
    got = ref_numpy.widen_bf16(run_attn(b, masks))
    assert (np.abs(got - want) <= BF16 * np.abs(want) + (BF16 + 2.0 ** -10) * size).all()


# ------------------------------------------------------------------------------------------------ verification
def run_verify(target, draft, tokens, parents, u, final, qsl, max_path, stride=0):
    n_seqs = len(qsl) - 1
    counts = torch.full((n_seqs + 1,), -5, dtype=torch.int32, device="cuda")
    path = torch.full((n_seqs + 1, max_path), -5, dtype=torch.int32, device="cuda")
    out = torch.full((n_seqs + 1, max_path + 1), -5, dtype=torch.int32, device="cuda")
    with B.Context(4, 1, 64, 16, 1, 1) as c:
        for _ in range(2):      # (the second call finds what the first left)
            B.ooco_verify_drafts(c.h, target, draft, dev(tokens), None if parents is None else dev(parents), dev(u), dev(final), dev(qsl), counts,
                                 path, out, max_path, n_seqs, len(tokens))
            torch.cuda.synchronize()
    assert (counts[n_seqs:] == -5).all() and (path[n_seqs:] == -5).all() and (out[n_seqs:] == -5).all()
    return counts[:-1].cpu().numpy(), path[:-1].cpu().numpy(), out[:-1].cpu().numpy()


def drafts(rng, nodes, V, chain, with_draft, dtype):
    qsl, par = starts(nodes), trees(nodes, rng, "chain" if chain else "random")
    T = len(par)
    z = rng.standard_normal((T, V)) * 3
    soft = lambda x: torch.from_numpy(np.exp(x) / np.exp(x).sum(-1, keepdims=True)).to(dtype)
    up = np.repeat(qsl[:-1], nodes) + np.maximum(par, 0)
    target, draft = soft(z), soft(z[up] + rng.standard_normal((T, V)) * 0.5) if with_draft else None
    # tokens among the likeliest after the parent, some twice, some no tokens at all
    order = np.argsort(-z[up], axis=1)
    tokens = order[np.arange(T), rng.integers(0, min(V, 4), T)].astype(np.int32)
    tokens[rng.random(T) < 0.03] = -1
    tokens[rng.random(T) < 0.03] = V
    return qsl, par, target, draft, tokens, rng.random(T).astype(np.float32), rng.random(len(nodes)).astype(np.float32)


@pytest.mark.parametrize("nodes, V, max_path", [([1], 1, 1), ([6] * 20, 1000, 5), ([64, 0, 3, 1, 17], 5003, 63), ([256, 300, 40], 777, 255),
                                                ([9] * 12, 20001, 3), ([5, 4], 40000, 0), ([3] * 300, 130, 2), ([12, 30], 70001, 29)],
                         ids=lambda x: f"{len(x)}-seqs" if isinstance(x, list) else str(x))
@pytest.mark.parametrize("form", ["tree", "chain", "chain with drafts"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_verify(nodes, V, max_path, form, dtype):
    rng = np.random.default_rng(V)
    qsl, par, target, draft, tokens, u, final = drafts(rng, nodes, V, form != "tree", form == "chain with drafts", dtype)
    say(f"case: verify {form} {dtype} nodes={nodes[:5]} V={V}")
    parents = par if form == "tree" else None
    want = S.verify_drafts(target.double().numpy(), None if draft is None else draft.double().numpy(), tokens, parents, u, final, qsl, max_path)
    got = run_verify(target.cuda(), None if draft is None else draft.cuda(), tokens, parents, u, final, qsl, max_path)
    say(f"  yields {want[0].mean():.2f}")
    for g, w in zip(got, want):
        assert (g == w).all()


def test_verify_rows_apart_and_at_odd_elements():
    rng = np.random.default_rng(8)
    qsl, par, target, draft, tokens, u, final = drafts(rng, [7, 5, 9], 3001, True, True, torch.float32)
    say("case: verify rows apart")
    want = S.verify_drafts(target.double().numpy(), draft.double().numpy(), tokens, None, u, final, qsl, 8)
    wide = torch.full((2, 21, 3010), float("nan"), device="cuda")
    wide[0, :, 3:3004], wide[1, :, 3:3004] = target.cuda(), draft.cuda()
    got = run_verify(wide[0, :, 3:3004], wide[1, :, 3:3004], tokens, None, u, final, qsl, 8)
    for g, w in zip(got, want):
        assert (g == w).all()


def test_verify_of_steps_without_rows():
    # the counts are the lengths' increments: they are written also where there is no row at all
    empty = lambda *shape: torch.empty(shape, device="cuda")
    i32 = lambda *shape: torch.full(shape, 9, dtype=torch.int32, device="cuda")
    say("case: verification without rows")
    with B.Context(4, 1, 64, 16, 1, 1) as c:
        for parents in (i32(0), None):
            counts, path, out = i32(3), i32(3, 4), i32(3, 5)
            c.verify_drafts(empty(0, 50), i32(0), empty(0), empty(3), torch.zeros(4, dtype=torch.int32, device="cuda"), counts, path, out, parents=parents)
            torch.cuda.synchronize()
            assert (counts == 0).all() and (path == -1).all() and (out == -1).all()


def test_verify_borders():
    # nothing left but the row itself, rows without weight, values that are no probabilities, random numbers at their ends
    V = 5000
    target = np.zeros((12, V), np.float32)
    draft = np.zeros((12, V), np.float32)
    tokens = np.zeros(12, np.int32)
    u, final = np.zeros(12, np.float32), np.zeros(6, np.float32)
    say("case: verify borders")
    target[0, 7], draft[1, 7], tokens[1], u[1] = 0.5, 1.0, 7, 0.75          # refused, p <= q everywhere: the draw is from p
    target[2, [10, 4999]], draft[3, 11], tokens[3], final[1] = 0.5, 1.0, 11, 1 - 2.0 ** -24   # never accepted; the last token
    draft[5, 3], tokens[5] = 1.0, 3                                          # a row of zeros: no token
    target[6, [1, 2, 3, 4]], tokens[7], u[7] = [np.nan, np.inf, -1.0, 0.25], 1, 0.5
    draft[7, 1] = 0.5                                                        # NaN is not accepted; only token 4 has weight
    target[8, 100], tokens[9], draft[9, 100] = 1.0, 100, 0.0                 # drawn from a distribution that says 0: accepted
    target[9, [20, 30]], final[4] = 0.5, 0.5                                 # exactly at the border: the later token
    target[10, 0], tokens[11], draft[11, 0], u[11] = 1.0, 0, 1.0, 1 - 2.0 ** -24
    target[11, 17] = 1e-30
    qsl = np.arange(0, 13, 2).astype(np.int32)
    want = S.verify_drafts(target.astype(np.float64), draft.astype(np.float64), tokens, None, u, final, qsl, 1)
    got = run_verify(torch.from_numpy(target).cuda(), torch.from_numpy(draft).cuda(), tokens, None, u, final, qsl, 1)
    for g, w in zip(got, want):
        assert (g == w).all()
    assert got[2].tolist() == [[7, -1], [4999, -1], [-1, -1], [4, -1], [100, 30], [0, 17]]


# ------------------------------------------------------------------------------------------------ accepted nodes to their places
@pytest.mark.parametrize("heads", [HEADS[0], HEADS[2], HEADS[3], HEADS[5]], ids=str)
@pytest.mark.parametrize("layers", [1, 3])
def test_compact(heads, layers):
    nodes, ctx = [20, 1, 64, 9, 40, 200, 0], [30, 5, 0, 15, 250, 77, 3]
    bs = [batch(heads, nodes, ctx, seed=500) for _ in range(layers)]
    rng = np.random.default_rng(layers)
    for x in bs:
        x.k_cache[:] = rng.integers(0, 65536, x.k_cache.shape)
        x.v_cache[:] = rng.integers(0, 65536, x.v_cache.shape)
    b = bs[0]
    max_path = 70
    path, counts = np.full((7, max_path), -1, np.int32), np.array([6, 1, 64, 4, 3, 71, 0], np.int32)
    for i in range(6):      # rising; nodes that stay, neighbours, places that other nodes of the path come from
        m = counts[i] - 1
        path[i, :m] = np.sort(rng.choice(np.arange(1, nodes[i]), m, replace=False)) if m else 0
    path[3, :3], path[4, :2] = [1, 2, 8], [2, 3]
    say(f"case: compact {heads} layers={layers}")
    d = [W.to_device(x) for x in bs]
    with context(b) as c:
        c.kv_compact([x.k_cache for x in d], [x.v_cache for x in d], dev(b.block_tables), dev(b.ctx_lens), dev(path), dev(counts))
        torch.cuda.synchronize()
    for x, y in zip(bs, d):
        S.kv_compact(x.k_cache, x.v_cache, b.block_tables, b.ctx_lens, path, counts)
        assert (bits(y.k_cache) == x.k_cache).all() and (bits(y.v_cache) == x.v_cache).all()


def test_compact_of_many_layers_and_nodes_without_a_place():
    heads, layers = (2, 1, 64), 230       # more layers than a launch takes
    b = batch(heads, [9, 9], [20, 40], seed=510)
    table = b.block_tables.copy()
    table[1, 3] = -1
    path, counts = np.array([[3, 5, 8, -1], [2, 7, 8, 9]], np.int32), np.array([4, 5], np.int32)
    cl = np.array([20, 16 * b.max_blocks_per_seq - 5], np.int32)
    say("case: compact many layers")
    k, v = bf16(np.stack([b.k_cache] * layers)), bf16(np.stack([b.v_cache] * layers))
    with context(b) as c:
        c.kv_compact(list(k), list(v), dev(table), dev(cl), dev(path), dev(counts))
        torch.cuda.synchronize()
    S.kv_compact(b.k_cache, b.v_cache, table, cl, path, counts)
    for i in (0, 111, 112, 223, 224, 229):
        assert (bits(k[i]) == b.k_cache).all() and (bits(v[i]) == b.v_cache).all()
    assert (k == k[0]).all() and (v == v[0]).all()


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals():
    say("case: refusals")
    i32 = torch.zeros(64, dtype=torch.int32, device="cuda")
    i64, f32 = torch.zeros(64, dtype=torch.int64, device="cuda"), torch.zeros(64, device="cuda")
    x = torch.zeros((4, 8, 64), dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros((4, 2, 8, 16, 8), dtype=torch.bfloat16, device="cuda")
    odd = torch.zeros(4 * 8 * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:]
    p = torch.ones((4, 8), device="cuda")
    EINVAL, ESHAPE, ENOMEM = B.OOCO_EINVAL, B.OOCO_ESHAPE, B.OOCO_ENOMEM

    def refused(status, text, call):
        with pytest.raises(B.OocoError) as e:
            call()
        assert e.value.status == status and text in e.value.message, e.value

    with B.Context(8, 2, 64, 16, 4, 2) as c:
        h = c.h
        for words in (0, 5):
            refused(ESHAPE, "mask_words", lambda: B.ooco_tree_masks(h, i32, i32, i32, i64, i32, words, 1, 4))
            refused(ESHAPE, "mask_words", lambda: B.ooco_attn_tree(h, x, kv, kv, i32, i32, i32, i64, words, x, 1, 4))
        refused(EINVAL, "NULL", lambda: B.ooco_tree_masks(h, None, i32, i32, i64, i32, 1, 1, 4))
        refused(EINVAL, "num_seqs", lambda: B.ooco_tree_masks(h, i32, i32, i32, i64, i32, 1, -1, 4))
        refused(EINVAL, "8-byte", lambda: B.ooco_tree_masks(h, i32, i32, i32, i32[1:], i32, 1, 1, 4))
        refused(EINVAL, "ooco_rope_set", lambda: c.rope_append(x, kv, kv, x, kv, kv, i32, i32, i32))
        for d in (0, 8, 24, 128):
            refused(ESHAPE, "rotary_dim", lambda: B.ooco_rope_set(h, d, 0, np.ones(d // 2)))
        refused(EINVAL, "finite", lambda: B.ooco_rope_set(h, 16, 0, np.full(8, np.nan)))
        refused(EINVAL, "factor", lambda: B.ooco_rope_set(h, 16, 0, np.ones(8), np.inf))
        refused(EINVAL, "NULL", lambda: B.ooco_rope_set(h, 16, 0, None))
        c.rope_set(np.ones(8))
        row = x[:, :2]
        good = dict(q=x, k=row, v=row, out=x)
        def rope(**kw):
            a = {**good, **kw}
            B.ooco_rope_append(h, a["q"], a["k"], a["v"], None, a["out"], kv, kv, i32, i32, i32, 1, 4)
        refused(EINVAL, "NULL", lambda: rope(q=None))
        refused(EINVAL, "16-byte", lambda: rope(k=odd[:512].view(4, 2, 64)))
        refused(EINVAL, "multiples of 8", lambda: rope(v=torch.zeros((4, 132), dtype=torch.bfloat16, device="cuda")[:, :128]))
        refused(EINVAL, "at least", lambda: rope(q=x.view(-1)[:4 * 128].view(4, 2, 64)))
        refused(EINVAL, "q_out is q", lambda: rope(q=torch.as_strided(x, (2, 8, 64), (1024, 64, 1)), out=x))
        with pytest.raises(ValueError):
            rope(q=x.transpose(1, 2))
        refused(EINVAL, "NULL", lambda: B.ooco_attn_tree(h, x, kv, kv, i32, i32, i32, None, 1, x, 1, 4))
        refused(EINVAL, "16-byte", lambda: B.ooco_attn_tree(h, odd[:2048], kv, kv, i32, i32, i32, i64, 1, x, 1, 4))
        def verify(**kw):
            a = {**dict(target=p, draft=None, parents=i32, u=f32, max_path=3, seqs=1), **kw}
            B.ooco_verify_drafts(h, a["target"], a["draft"], i32, a["parents"], a["u"], f32, i32, i32, i32, i32, a["max_path"], a["seqs"], 4)
        refused(EINVAL, "chains", lambda: verify(draft=p))
        refused(EINVAL, "NULL", lambda: verify(u=None))
        refused(EINVAL, "max_path", lambda: verify(max_path=-1))
        refused(EINVAL, "vocab", lambda: verify(target=p[:, :0]))
        refused(ENOMEM, "sequences", lambda: verify(seqs=2 ** 20))
        for bad in (dict(target=p.half()), dict(target=p.t()), dict(draft=p.bfloat16(), parents=None), dict(draft=torch.ones((4, 9), device="cuda")[:, :8], parents=None)):
            with pytest.raises(ValueError):
                verify(**bad)
        refused(EINVAL, "NULL", lambda: B.ooco_kv_compact(h, [kv], [None], i32, i32, i32, i32, 3, 1))
        refused(EINVAL, "16-byte", lambda: B.ooco_kv_compact(h, [kv], [odd], i32, i32, i32, i32, 3, 1))
        refused(EINVAL, "max_path", lambda: B.ooco_kv_compact(h, [kv], [kv], i32, i32, i32, i32, -3, 1))
        with pytest.raises(ValueError):
            B.ooco_kv_compact(h, [kv, kv], [kv], i32, i32, i32, i32, 3, 1)
        for call in (lambda n, t: B.ooco_tree_masks(h, i32, i32, i32, i64, i32, 1, n, t), lambda n, t: B.ooco_attn_tree(h, x, kv, kv, i32, i32, i32, i64, 1, x, n, t)):
            call(0, 4)      # nothing to do
            call(1, 0)
        B.ooco_kv_compact(h, [], [], i32, i32, i32, i32, 3, 1)
    with B.Context(8, 2, 64, 16, 4, 2, workspace_bytes=256) as c:
        refused(ENOMEM, "workspace", lambda: B.ooco_attn_tree(c.h, x, kv, kv, i32, i32, i32, i64, 1, x, 1, 4))
        refused(ENOMEM, "workspace", lambda: B.ooco_verify_drafts(c.h, torch.ones((4, 10 ** 6), device="cuda"), None, i32, None, f32, f32, i32, i32,
                                                                  i32, i32, 3, 1, 4))
