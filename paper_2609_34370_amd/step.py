"""One verification step on the GPU: append -> verify attention -> accept.

Holds the device buffers of a batch (metadata, pools, outputs, workspaces sized once from the
library's queries) and calls the three entry points of libspexis in order on one stream.

Options: a cache held in 8 bits (AttentionInputs8 in place of AttentionInputs), q and keys that the append
rotates by position (rotary), the emitted tokens' log probabilities behind the acceptance (top_logprobs), prefixes
that sequences share (shared), and the attention weights that a later eviction goes by (weights).

Without acceptance (acc None) the step is that of prompts, of any length: append and attention.
"""
from __future__ import annotations

import math
from typing import Optional, Union

import numpy as np
import torch

from . import spexis as sx
from .workloads import AcceptInputs, AttentionInputs, AttentionInputs8, Batch, RotaryInputs


class VerifyStep:
    def __init__(self, batch: Batch, attn: Union[AttentionInputs, AttentionInputs8], acc: Optional[AcceptInputs],
                 kv_chunk_tokens: int = 0, kind: int = sx.SPEXIS_INPUT_LOGITS, device="cuda",
                 rotary: Optional[RotaryInputs] = None, top_logprobs: Optional[int] = None, shared: Optional[tuple] = None,
                 weights: Optional[torch.Tensor] = None, positions: Optional[np.ndarray] = None):
        """rotary: attn's q and new_k are not rotated yet; the append does it (the rotated q is self.q).
        top_logprobs: with acceptance from logits, the emitted tokens' log probabilities and entropies, and that many
        alternatives of each (0: none); self.logprob, entropy [B][max_k+1], top_ids, top_logprob
        [B][max_k+1][top_logprobs].
        positions [T]: where the rotation turns the tokens to, if not to their places in the cache (after an eviction).
        shared: (group_start_loc, prefix_lens) of sequences that begin with the same blocks.
        weights [num_blocks][Hkv][block_size] fp32: the sums of the cached keys' attention weights, to which the step adds
        those of its accepted tokens (of all tokens without acceptance); bf16 cache only.  Shared keys have none.
        With shared or weights, or more than 64 query rows a KV head, the attention is that of prompts (weights need its lse;
        workload 2: 146 us for the verification attention's 128), which cuts keys by itself: kv_chunk_tokens is not used."""
        spec = batch.spec
        self.batch, self.spec, self.kind = batch, spec, kind
        self.kv_chunk_tokens = kv_chunk_tokens
        dev = torch.device(device)
        self.qsl = torch.as_tensor(batch.qsl, device=dev)
        self.seq_lens = torch.as_tensor(batch.seq_lens, device=dev)
        self.tables = torch.as_tensor(batch.block_tables, device=dev)
        self.attn = attn
        self.in8 = isinstance(attn, AttentionInputs8)
        self.positions = None
        if positions is not None:
            if rotary is None:
                raise ValueError("positions without a rotation")
            positions = np.asarray(positions, np.int32)
            if positions.min() < 0 or positions.max() >= rotary.cos_sin.shape[0]:
                raise ValueError(f"the rotation's table ends at position {rotary.cos_sin.shape[0]}, "
                                 f"the tokens at {positions.max()}")
            self.positions = torch.as_tensor(positions, device=dev)
        elif rotary is not None and rotary.cos_sin.shape[0] < batch.max_seq_len:
            raise ValueError(f"the rotation's table ends at position {rotary.cos_sin.shape[0]}, "
                             f"the longest sequence at {batch.max_seq_len}")
        self.rotary = rotary
        self.q = attn.q if rotary is None else torch.empty_like(attn.q)
        self.out = torch.empty_like(attn.q)
        self.scale = 1.0 / math.sqrt(spec.head_dim)
        if weights is not None and self.in8:
            raise ValueError("attention weights are kept for a bf16 cache")
        self.weights = weights
        if shared is not None:
            for start, end, n in zip(shared[0], shared[0][1:], shared[1]):
                blocks = batch.block_tables[start:end, : n // spec.block_size]
                if (batch.ctx_lens[start:end] < n).any() or (blocks != blocks[:1]).any():
                    raise ValueError(f"sequences {start} to {end - 1} do not share {n} cached tokens")
        self.shared = None if shared is None else tuple(torch.as_tensor(x, dtype=torch.int32, device=dev) for x in shared)
        heads = (spec.num_q_heads, spec.num_kv_heads, spec.head_dim)
        # more rows a KV head than the verification attention takes, and what it does not give
        self.tiles = (shared is not None or weights is not None or
                      spec.num_q_heads // spec.num_kv_heads * batch.max_query_len > 64)
        if self.shared is not None:
            ws = sx.spexis_shared_attention_workspace_size(batch.B, len(self.shared[1]), *heads, batch.T, batch.max_query_len,
                                                           batch.max_seq_len)
        elif self.tiles:
            ws = sx.spexis_prompt_attention_workspace_size(batch.B, *heads, batch.T, batch.max_query_len, batch.max_seq_len)
        else:
            size = sx.spexis_verify_attention_kv8_workspace_size if self.in8 else sx.spexis_verify_attention_workspace_size
            ws = size(batch.B, *heads, batch.max_query_len, batch.max_seq_len, kv_chunk_tokens)
        self.attn_ws = torch.empty(max(ws, 16), dtype=torch.uint8, device=dev)
        self.lse = self.first_keys = None
        if weights is not None:
            self.lse = torch.empty(attn.q.shape[:2], device=dev)
            # the lengths after the step (with acceptance, without the rejected tokens) and after an eviction
            self.lens_after, self.lens_evicted = self.seq_lens.clone(), torch.empty_like(self.seq_lens)
            ws = sx.spexis_evict_kv_workspace_size(batch.B, spec.num_kv_heads, batch.max_seq_len)
            self.evict_ws = torch.empty(max(ws, 16), dtype=torch.uint8, device=dev)
            if shared is not None:   # the keys that every sequence shares, in whole blocks
                first = np.zeros(batch.B, np.int32)
                for start, end, n in zip(shared[0], shared[0][1:], shared[1]):
                    first[start:end] = n // spec.block_size * spec.block_size
                self.first_keys = torch.as_tensor(first, device=dev)
        self.acc = acc
        self.max_k = batch.max_k
        if acc is not None:
            aw = sx.spexis_accept_workspace_size(batch.B, spec.vocab, self.max_k)
            self.acc_ws = torch.empty(aw, dtype=torch.uint8, device=dev)
            self.accepted_len = torch.empty(batch.B, dtype=torch.int32, device=dev)
            self.out_tokens = torch.empty((batch.B, self.max_k + 1), dtype=torch.int32, device=dev)
            self.row_status = torch.empty(batch.B, dtype=torch.int32, device=dev)
        self.top_logprobs = top_logprobs
        if top_logprobs is not None:
            if acc is None or kind != sx.SPEXIS_INPUT_LOGITS:
                raise ValueError("log probabilities need acceptance from logits")
            items = (batch.B, self.max_k + 1)
            # the logit row of every place in out_tokens (places past a sequence's drafts hold no token)
            j = np.minimum(np.arange(self.max_k + 1)[None, :], np.asarray(batch.k)[:, None])
            self.rows = torch.as_tensor((batch.qsl[:-1, None] + j).astype(np.int32), device=dev)
            self.logprob = torch.empty(items, device=dev)
            self.entropy = torch.empty(items, device=dev)
            self.top_ids = torch.empty((*items, top_logprobs), dtype=torch.int32, device=dev)
            self.top_logprob = torch.empty((*items, top_logprobs), device=dev)
            lw = sx.spexis_token_logprobs_workspace_size(items[0] * items[1], spec.vocab, top_logprobs)
            self.lp_ws = torch.empty(max(lw, 16), dtype=torch.uint8, device=dev)

    def _cache(self):
        """The cache's pools (and scales), and where the batch lies in it."""
        s, b, a = self.spec, self.batch, self.attn
        pools = (a.k_pool, a.v_pool, a.scales) if self.in8 else (a.k_pool, a.v_pool)
        return (*pools, b.num_blocks, s.num_kv_heads, s.block_size, s.head_dim, self.qsl, self.seq_lens, self.tables, b.T,
                b.max_query_len)

    def append(self, stream=None):
        new = (self.attn.new_k, self.attn.new_v)
        rotation = {}
        if self.rotary is not None:
            rotation = dict(cos_sin=self.rotary.cos_sin, style=self.rotary.style, positions=self.positions,
                            q=self.attn.q, q_out=self.q)
        if self.in8:
            sx.spexis_rotate_append_kv8(*self._cache(), *new, **rotation, stream=stream)
        elif rotation:
            sx.spexis_rotate_append_kv(*self._cache(), *new, **rotation, stream=stream)
        else:
            sx.spexis_append_kv(*self._cache(), *new, stream=stream)

    def attention(self, stream=None):
        if self.tiles:
            rows = (self.q, self.spec.num_q_heads, self.scale, self.out, self.attn_ws)
            if self.shared is not None:
                f = sx.spexis_shared_attention_kv8 if self.in8 else sx.spexis_shared_attention
                f(*self._cache(), self.batch.max_seq_len, *self.shared, *rows, lse=self.lse, stream=stream)
            else:
                f = sx.spexis_prompt_attention_kv8 if self.in8 else sx.spexis_prompt_attention
                f(*self._cache(), self.batch.max_seq_len, *rows, lse=self.lse, stream=stream)
            return
        f = sx.spexis_verify_attention_kv8 if self.in8 else sx.spexis_verify_attention
        f(*self._cache(), self.batch.max_seq_len, self.q, self.spec.num_q_heads, self.scale, self.out, self.attn_ws,
          kv_chunk_tokens=self.kv_chunk_tokens, stream=stream)

    def _begin_lens(self, stream):
        """self.lens_after with the step's new tokens, rejected ones among them."""
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            self.lens_after.copy_(self.seq_lens)

    def accept(self, target=None, draft=None, kind=None, stream=None, seq_lens_inout=None):
        """seq_lens_inout: the lengths that lose the rejected tokens; self.lens_after of a step with weights."""
        a = self.acc
        if self.weights is not None and seq_lens_inout is None:
            self._begin_lens(stream)
            seq_lens_inout = self.lens_after
        kind = self.kind if kind is None else kind
        target = a.target_logits if target is None else target
        draft = a.draft_logits if draft is None else draft
        sx.spexis_accept(kind, self.qsl, target, draft, a.draft_ids, a.u_accept, a.u_sample, self.max_k,
                         self.accepted_len, self.out_tokens, self.row_status, self.acc_ws,
                         temperature=a.temperature, seq_lens_inout=seq_lens_inout, stream=stream)

    def logprobs(self, stream=None):
        """Of the tokens that the acceptance emitted."""
        sx.spexis_token_logprobs(self.acc.target_logits, self.out_tokens, self.logprob, self.lp_ws, row_ids=self.rows,
                                 entropy=self.entropy, top_ids=self.top_ids, top_logprobs=self.top_logprob,
                                 temperature=self.acc.temperature, stream=stream)

    def add_weights(self, stream=None):
        """To self.weights, those of the accepted tokens, by the lengths after the step (self.lens_after, of the acceptance)."""
        s, b, a = self.spec, self.batch, self.attn
        if self.acc is None:
            self._begin_lens(stream)
        sx.spexis_attention_weights(a.k_pool, b.num_blocks, s.num_kv_heads, s.block_size, s.head_dim, self.qsl, self.lens_after,
                                    self.tables, b.T, b.max_query_len, b.max_seq_len, self.q, s.num_q_heads, self.scale, self.lse,
                                    self.weights, weights_in=self.weights,
                                    accepted_len=self.accepted_len if self.acc is not None else None,
                                    first_keys=self.first_keys, stream=stream)

    def evict(self, keep_lens, keep_last, stream=None) -> torch.Tensor:
        """Behind the step, drops all but keep_lens keys of each sequence, those of least weight; shared keys and the last
        keep_last stay.  The new lengths (self.lens_evicted), from which another eviction before the next step goes on."""
        s, b, a = self.spec, self.batch, self.attn
        if self.weights is None:
            raise ValueError("no attention weights to go by")
        sx.spexis_evict_kv(a.k_pool, a.v_pool, self.weights, b.num_blocks, s.num_kv_heads, s.block_size, s.head_dim,
                           self.lens_after, self.tables, b.max_seq_len, keep_lens, keep_last, self.weights,
                           self.lens_evicted, self.evict_ws, first_keys=self.first_keys, stream=stream)
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            self.lens_after.copy_(self.lens_evicted)
        return self.lens_evicted

    def run(self, stream=None):
        self.append(stream)
        self.attention(stream)
        if self.acc is not None:
            self.accept(stream=stream)
        if self.weights is not None:
            self.add_weights(stream)
        if self.top_logprobs is not None:
            self.logprobs(stream)

    def capture(self, warmup: int = 1):
        """Records run() into a HIP graph (torch.cuda.CUDAGraph); replay() then launches the whole
        step at once.  Every buffer is allocated in __init__ and the library calls neither
        allocate nor set memory (the acceptance counters are cleared by its first kernel), so the
        graph holds only the step's kernel launches.  A replay reads the current contents of the
        input buffers; the sizes are those of this batch.  The warm-up's attention weights do not count."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            before = self.weights.clone() if self.weights is not None else None
            for _ in range(warmup):
                self.run()
            if before is not None:
                self.weights.copy_(before)
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.run()
        return self.graph

    def replay(self):
        self.graph.replay()

    def accept_outputs(self):
        return (self.accepted_len.cpu().numpy(), self.out_tokens.cpu().numpy(), self.row_status.cpu().numpy())


def bf16_to_u16(t: torch.Tensor) -> np.ndarray:
    """Host uint16 view of a bf16 tensor's bits (for the oracle)."""
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)
