"""A step of speculative decoding over the layers of a model, built on the library's calls only: masks and positions of the drafted
trees once per step, rotary positions, append and attention layer by layer, then the verification, whose accepted nodes are moved to
their places in the caches of all layers.  Lengths stay on the device: no call of a step waits for the GPU, and a step can be recorded
into a HIP graph and replayed with other trees, lengths and random numbers in the same tensors.

Data movement only; every number is computed by the library's kernels (the lengths are advanced by one addition of torch).
"""
from __future__ import annotations

import torch


class TreeStep:
    """Buffers of a step for up to `rows` nodes of `seqs` sequences; `ctx` is a binding.Context with its rotation set.

    begin(...) once per step, layer(...) for every layer, finish(...) once; tensors as in include/ooco.h, and rows, sequences and layers
    as many as the tensors given hold.  The buffers are the step's until finish() has run on its stream."""

    def __init__(self, ctx, rows, seqs, Hq, head_dim, mask_words=1, max_path=16, device="cuda"):
        new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=device)
        self.ctx = ctx
        self._masks, self._positions = new((rows, mask_words), torch.int64), new(rows, torch.int32)
        self._q, self._out = (new((rows, Hq, head_dim), torch.bfloat16) for _ in range(2))
        self._counts, self._path, self._tokens = new(seqs, torch.int32), new((seqs, max_path), torch.int32), new((seqs, max_path + 1), torch.int32)
        self._step = None

    def begin(self, parents, query_start_loc, ctx_lens, block_tables):
        T, B = parents.shape[0], ctx_lens.shape[0]
        if T > self._positions.shape[0] or B > self._counts.shape[0]:
            raise ValueError(f"{T} nodes of {B} sequences: the step has room for {self._positions.shape[0]} of {self._counts.shape[0]}")
        self._step = (parents, query_start_loc, ctx_lens, block_tables)
        self.masks, self.positions = self._masks[:T], self._positions[:T]
        self.ctx.tree_masks(parents, query_start_loc, ctx_lens, self.masks, self.positions)

    def layer(self, q, k_new, v_new, k_cache, v_cache):
        """Attention output [rows][Hq][head_dim] of a layer; the next layer's call reuses its buffer."""
        _, qsl, cl, table = self._step
        rotated, out = self._q[:q.shape[0]], self._out[:q.shape[0]]
        self.ctx.rope_append(q, k_new, v_new, rotated, k_cache, v_cache, table, qsl, cl, positions=self.positions)
        self.ctx.attn_tree(rotated, k_cache, v_cache, table, qsl, cl, self.masks, out)
        return out

    def finish(self, target_probs, tokens, uniforms, final_uniforms, k_caches, v_caches):
        """Verifies the nodes, moves the accepted ones and advances ctx_lens (in place) by what each sequence has gained.
        Returns counts [seqs] and tokens [seqs][max_path + 1] (see ooco_verify_drafts); the last of a sequence's `counts` tokens is the
        root of its next tree."""
        parents, qsl, cl, table = self._step
        B = cl.shape[0]
        counts, path, out_tokens = self._counts[:B], self._path[:B], self._tokens[:B]
        self.ctx.verify_drafts(target_probs, tokens, uniforms, final_uniforms, qsl, counts, path, out_tokens, parents=parents)
        self.ctx.kv_compact(k_caches, v_caches, table, cl, path, counts)
        cl.add_(counts)
        return counts, out_tokens
