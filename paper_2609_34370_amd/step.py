"""One verification step on the GPU: append -> verify attention -> accept.

Holds the device buffers of a batch (metadata, pools, outputs, workspaces sized once from the
library's queries) and calls the three entry points of libspexis in order on one stream.

Options: a cache held in 8 bits (AttentionInputs8 in place of AttentionInputs), q and keys that the append
rotates by position (rotary), and the emitted tokens' log probabilities behind the acceptance (top_logprobs).
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
                 rotary: Optional[RotaryInputs] = None, top_logprobs: Optional[int] = None):
        """rotary: attn's q and new_k are not rotated yet; the append does it (the rotated q is self.q).
        top_logprobs: with acceptance from logits, the emitted tokens' log probabilities and entropies, and that many
        alternatives of each (0: none); self.logprob, entropy [B][max_k+1], top_ids, top_logprob
        [B][max_k+1][top_logprobs]."""
        spec = batch.spec
        self.batch, self.spec, self.kind = batch, spec, kind
        self.kv_chunk_tokens = kv_chunk_tokens
        dev = torch.device(device)
        self.qsl = torch.as_tensor(batch.qsl, device=dev)
        self.seq_lens = torch.as_tensor(batch.seq_lens, device=dev)
        self.tables = torch.as_tensor(batch.block_tables, device=dev)
        self.attn = attn
        self.in8 = isinstance(attn, AttentionInputs8)
        if rotary is not None and rotary.cos_sin.shape[0] < batch.max_seq_len:
            raise ValueError(f"the rotation's table ends at position {rotary.cos_sin.shape[0]}, "
                             f"the longest sequence at {batch.max_seq_len}")
        self.rotary = rotary
        self.q = attn.q if rotary is None else torch.empty_like(attn.q)
        self.out = torch.empty_like(attn.q)
        self.scale = 1.0 / math.sqrt(spec.head_dim)
        size = sx.spexis_verify_attention_kv8_workspace_size if self.in8 else sx.spexis_verify_attention_workspace_size
        ws = size(batch.B, spec.num_q_heads, spec.num_kv_heads, spec.head_dim, batch.max_query_len, batch.max_seq_len,
                  kv_chunk_tokens)
        self.attn_ws = torch.empty(max(ws, 16), dtype=torch.uint8, device=dev)
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
            rotation = dict(cos_sin=self.rotary.cos_sin, style=self.rotary.style, q=self.attn.q, q_out=self.q)
        if self.in8:
            sx.spexis_rotate_append_kv8(*self._cache(), *new, **rotation, stream=stream)
        elif rotation:
            sx.spexis_rotate_append_kv(*self._cache(), *new, **rotation, stream=stream)
        else:
            sx.spexis_append_kv(*self._cache(), *new, stream=stream)

    def attention(self, stream=None):
        f = sx.spexis_verify_attention_kv8 if self.in8 else sx.spexis_verify_attention
        f(*self._cache(), self.batch.max_seq_len, self.q, self.spec.num_q_heads, self.scale, self.out, self.attn_ws,
          kv_chunk_tokens=self.kv_chunk_tokens, stream=stream)

    def accept(self, target=None, draft=None, kind=None, stream=None, seq_lens_inout=None):
        a = self.acc
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

    def run(self, stream=None):
        self.append(stream)
        self.attention(stream)
        if self.acc is not None:
            self.accept(stream=stream)
        if self.top_logprobs is not None:
            self.logprobs(stream)

    def capture(self, warmup: int = 1):
        """Records run() into a HIP graph (torch.cuda.CUDAGraph); replay() then launches the whole
        step at once.  Every buffer is allocated in __init__ and the library calls neither
        allocate nor set memory (the acceptance counters are cleared by its first kernel), so the
        graph holds only the step's kernel launches.  A replay reads the current contents of the
        input buffers; the sizes are those of this batch."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(warmup):
                self.run()
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
