"""Decoding rounds: the paged cache of a batch of sequences, from one verification to the next.

A round feeds every sequence a chunk of new tokens (its last token and K drafted ones, or a prompt), attends from them
over what is cached, and ends with the verification of the drafts, whose accept lengths decide what stays cached (prompts
and chunks with fewer drafts may be among them)::

    state = DecodeRounds(B, layers, n_blocks, block_size, kv_heads, head_dim, max_blocks)
    plan = state.begin(prompt_lens, rows)            # rows: the host's bound for the sum of the lengths
    for layer in range(layers):
        o = state.attend(layer, q, k, v)             # appends k and v to the cache, attends over it
    state.keep_all()                                 # a prompt is kept whole
    while ...:
        plan = state.begin(chunk_lens, rows)         # lengths, blocks and slots follow from the accept lengths on the GPU
        for layer in range(layers):
            o = state.attend(layer, q, k, v)
        accept_len, tokens, groups, flags = state.verify(target_logits, draft_logits, draft_tokens, handle, uniforms)

Nothing here waits for the GPU: lengths stay there from round to round.  A call runs on its ``stream``, or on the current
one; where that is another one than the last call's, it is put behind it, so that a round may use several (what a graph
replays is the caller's to order).  What a call reads has to be complete on its stream.  The arithmetic is the library's
(``pcg_cache_plan``, ``pcg_cache_append``, ``pcg_cache_attention``, ``pcg_prompt_attention``, ``pcg_verify``; with positions
``pcg_cache_append_rotary``; with 4 bits ``pcg_cache_append_fourbit`` and ``pcg_cache_attention_fourbit``).
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import Optional

import torch

from . import binding


class DecodeRounds:
    """Cache, block tables and lengths of ``B`` sequences (rows of a batch; a finished one's row is free for another).

    ``n_blocks`` blocks of ``block_size`` tokens are shared by all sequences and all layers' caches alike; a sequence
    holds ``max_blocks`` at most.

    ``rotary``: a table [positions, dim] float32 of the cosines, then the sines, of each position's angles; queries and keys
    are then turned by the angles of their tokens' positions (pairs of adjacent dimensions where ``interleaved``); at a position
    that the table does not have they become NaN.
    ``fourbit``: the cache holds 4.5 bits a value, with ``k_scale`` and ``v_scale`` as ``pcg_cache_append_fourbit`` says;
    ``dtype`` is then not used, q, k and v may be of any type."""

    def __init__(self, B: int, layers: int, n_blocks: int, block_size: int, kv_heads: int, head_dim: int, max_blocks: int,
                 dtype=torch.bfloat16, device="cuda", rotary=None, interleaved: bool = False, fourbit: bool = False, k_scale: float = 1.0,
                 v_scale: float = 1.0):
        if min(B, layers, n_blocks, max_blocks) < 1:
            raise ValueError("B, layers, n_blocks and max_blocks must be at least 1")

        def ints(*shape, fill=0):
            return torch.full(shape, fill, dtype=torch.int32, device=device)

        self.k_cache = self.v_cache = self.cache = None
        if fourbit:
            shape = (layers, *binding.pcg_fourbit_cache_shape(n_blocks, kv_heads, block_size, head_dim))
            self.cache = torch.empty(shape, dtype=torch.uint8, device=device)
        else:
            shape = (layers, n_blocks, kv_heads, block_size, head_dim)
            self.k_cache = torch.empty(shape, dtype=dtype, device=device)
            self.v_cache = torch.empty(shape, dtype=dtype, device=device)
        self.rotary, self.interleaved, self._scales = rotary, interleaved, dict(k_scale=k_scale, v_scale=v_scale)
        self.block_size, self.B = block_size, B
        self.block_table = ints(B, max_blocks, fill=-1)
        self.free_ring = torch.arange(n_blocks, dtype=torch.int32, device=device)
        self.ring_state = torch.tensor([0, n_blocks], dtype=torch.int32, device=device)
        self.cached_len, self.held = ints(B), ints(B)
        self.accept_len = ints(B, fill=-1)  # of the last round; -1: none of its tokens stays
        self.plan: Optional[binding.CachePlan] = None
        self._workspace = None
        # of the last call; there is none for a state in host memory, of which the lengths can be followed without a GPU
        self._device = self.cached_len.get_device()
        self._stream = torch.cuda.current_stream(self._device) if self.cached_len.is_cuda else None
        self._at = None if self._stream is None else self._stream.cuda_stream

    def _behind(self, stream):
        """The given stream of a call, or None where that is the current one.  A stream that the last call was not on waits
        for it, and the state's memory is not given out again before that stream, too, is done with it."""
        if self._stream is None:
            return None
        dev = self._device
        at = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
        stream = None if stream is None else binding._beside(stream, dev)
        if at != self._at:
            last, self._stream, self._at = self._stream, stream or torch.cuda.current_stream(dev), at
            if not torch.cuda.is_current_stream_capturing():  # a captured call cannot wait for what is not in the graph
                self._stream.wait_stream(last)
            binding._lend(self._stream, self.cached_len, self.held, self.ring_state, self.accept_len, self.block_table, self.free_ring,
                          self.k_cache, self.v_cache, self.cache, self.rotary, self._workspace)
        return stream

    def _on(self, stream):
        return nullcontext() if stream is None else torch.cuda.stream(stream)

    def begin(self, new_len, rows: int, stream=None) -> binding.CachePlan:
        """Plans a round of ``new_len`` [B] new tokens a sequence (int32, on the device; negative: the sequence has
        finished and its blocks are free again), packed into ``rows`` rows at the most.  ``plan.row_start`` and
        ``plan.positions`` say which row is which token; a sequence with ``plan.flags`` set has no part in the round."""
        if self.plan is not None:
            raise RuntimeError("the last round has not ended: verify() or keep_all()")
        stream = self._behind(stream)
        plan = binding.pcg_cache_plan(self.cached_len, new_len, self.held, self.block_table, self.free_ring, self.ring_state,
                                      self.block_size, rows, accept_len=self.accept_len, stream=stream)
        self.plan = plan
        self.cached_len, self.held, self.ring_state = plan.cached_len, plan.held, plan.ring_state
        return plan

    def attend(self, layer: int, q, k, v, scale: Optional[float] = None, fresh: bool = False, out=None, stream=None):
        """One layer's attention of the round's rows: q [rows, q_heads, head_dim], k and v [rows, kv_heads, head_dim].

        Writes k and v to the cache first, where the state has a rotation turned with q.  ``fresh`` says that no sequence has
        anything cached, and every one of the round's was given its blocks: the rows' own keys and values are then read instead
        of the cache (as it holds them, where that is in 4 bits)."""
        if self.plan is None:
            raise RuntimeError("no round has begun")
        plan = self.plan
        rows = plan.slots.shape[0]
        if q.shape[0] != rows or k.shape[0] != rows:  # fewer would cut sequences short, whose rows then see fewer keys
            raise ValueError(f"the round has {rows} rows; q has {q.shape[0]}, k {k.shape[0]}")
        stream = self._behind(stream)
        if self._workspace is None:
            need = binding.pcg_attention_workspace_bytes(self.B, q.shape[1], k.shape[1], q.shape[2], binding.dtype_code(q))
            self._workspace = binding._empty(self.cached_len, need, torch.uint8, stream)
        turned = self.rotary is not None
        if self.cache is not None:
            cache, k_out, v_out = self.cache[layer], None, None
            if fresh:
                k_out, v_out = (binding._empty(t, t.shape, t.dtype, stream) for t in (k, v))
            q_turned = binding.pcg_cache_append_fourbit(q if turned else None, k, v, plan.slots, cache, k_out=k_out, v_out=v_out, stream=stream,
                                                        positions=plan.positions if turned else None, table=self.rotary,
                                                        interleaved=self.interleaved, **self._scales)
            q, k, v = q_turned if turned else q, k_out, v_out
        elif turned:
            kc, vc = self.k_cache[layer], self.v_cache[layer]
            k_out = binding._empty(k, k.shape, k.dtype, stream) if fresh else None
            q = binding.pcg_cache_append_rotary(q, k, v, plan.slots, plan.positions, self.rotary, kc, vc, interleaved=self.interleaved,
                                                k_out=k_out, stream=stream)
            k = k_out
        else:
            kc, vc = self.k_cache[layer], self.v_cache[layer]
            binding.pcg_cache_append(k, v, plan.slots, kc, vc, stream=stream)
        if fresh:
            return binding.pcg_prompt_attention(q, k, v, plan.row_start, scale=scale, out=out, workspace=self._workspace, stream=stream)
        if self.cache is not None:
            return binding.pcg_cache_attention_fourbit(q, plan.row_start, plan.kv_len, self.block_table, cache, scale=scale, out=out,
                                                       workspace=self._workspace, stream=stream, **self._scales)
        return binding.pcg_cache_attention(q, plan.row_start, plan.kv_len, self.block_table, kc, vc, scale=scale, out=out,
                                           workspace=self._workspace, stream=stream)

    def verify(self, target_logits, draft_logits, draft_tokens, groups, uniforms, temperature: float = 1.0, whole=None, stream=None, **kw):
        """``pcg_verify`` of the round's drafts: all ``B`` sequences, K drafted tokens each.

        Of a chunk its first token and the accepted drafts stay cached; of one with fewer than K drafts, those that it
        has.  A chunk of more than K + 1 tokens is a prompt and stays whole, and so do the chunks of the sequences that
        ``whole`` [B] (bool, on the device) names: short prompts.  What is returned is ``pcg_verify``'s, of K drafts for
        every sequence: a prompt's part of it means nothing, nor do accepted drafts beyond those that a chunk has."""
        if self.plan is None:
            raise RuntimeError("no round has begun")
        if draft_tokens.dim() != 2 or draft_tokens.shape[0] != self.B:
            raise ValueError(f"the round is verified as a batch of all {self.B} sequences: draft_tokens must be [B, K]")
        if whole is not None and (whole.shape != (self.B,) or whole.dtype is not torch.bool or whole.device != self.cached_len.device):
            raise ValueError("whole must be a bool tensor [B] on the state's device")
        stream = self._behind(stream)
        result = binding.pcg_verify(target_logits, draft_logits, draft_tokens, groups, uniforms, temperature, stream=stream, **kw)
        if whole is not None and stream is not None:
            whole.record_stream(stream)
        with self._on(stream):
            last = self._last()
            prompt = last > draft_tokens.shape[1]
            self._end(torch.where(prompt if whole is None else prompt | whole, last, result[0]), last)
        return result

    def keep_all(self, stream=None):
        """Ends a round without drafts (a prompt, or a chunk of one): all of its tokens stay cached."""
        if self.plan is None:
            raise RuntimeError("no round has begun")
        with self._on(self._behind(stream)):
            last = self._last()
            self._end(last, last)

    def _last(self):
        """Number of the last token that each sequence fed, by the plan (the caller's lengths may be the next round's by
        now); below 0 where it fed none, as a flagged or finished one."""
        return self.plan.kv_len - self.plan.cached_len - 1

    def _end(self, accept_len, last=None):
        # no more than was fed stays
        self.accept_len = torch.minimum(accept_len, self._last() if last is None else last).clamp(min=-1)
        self.plan = None
