"""The outer loop of speculative decoding (Algorithm 3) for models that attend to their context, on the library's paged
key-value cache.

    python -m paper_2403_10444_b200.specdec --context 512 [--V 32768] [--B 64] [--gammas 2,4,8] [--iterations 32] [--window 0 --sinks 0]

Two synthetic decoders (``workloads.attention_models``: token embedding, causal attention layers, unembedding; no weights of any
real model) take the place of the two tables of ``specdec.run``.  Each keeps its keys and values in a cache of its own.  An iteration
extends both caches by gamma + 1 tokens (``bv_pages_extend``), drafts gamma tokens one at a time, scores the block with one pass of the target over its
gamma + 1 tokens (``bv_cache_append``, ``bv_cache_attend`` in every layer), verifies it, and takes what was not accepted out of
both caches (``bv_pages_truncate`` with the verification's out_len).  Projections are torch products; attention, bookkeeping,
sampling and verification run in the CUDA library.
"""
from __future__ import annotations

from typing import Dict, List

import torch

from . import binding as bv


class PagedCache:
    """The key-value cache of one model: ``layers`` pools of pages, one table.  Every page is free at first."""

    def __init__(self, layers: int, B: int, capacity: int, heads: int, D: int, page_size: int, dtype, device, spare: int = 0):
        width = -(-capacity // page_size)
        self.page_size = page_size
        self.k: List[torch.Tensor] = [torch.zeros((B * width + spare, heads, page_size, D), dtype=dtype, device=device) for _ in range(layers)]
        self.v = [torch.zeros_like(x) for x in self.k]
        i32 = dict(dtype=torch.int32, device=device)
        self.table = torch.full((B, width), -1, **i32)
        self.lens = torch.zeros((B,), **i32)
        self.refs = torch.zeros((B * width + spare,), **i32)

    def extend(self, n: int, n_new=None) -> torch.Tensor:
        """Room for n (n_new[b]) more tokens of each sequence; pages that were shared are copied.  Returns the tokens there is room for,
        -1 where there is none."""
        new, copies = bv.bv_pages_extend(self.table, self.lens, self.refs, self.page_size, n, n_new)
        for k, v in zip(self.k, self.v):
            bv.bv_pages_copy(k, v, copies)
        return new

    def truncate(self, keep: torch.Tensor, n: int = 0, n_new=None) -> None:
        """The first keep[b] of the n newest tokens (n = 0: of all) stay."""
        bv.bv_pages_truncate(self.table, self.lens, self.refs, self.page_size, keep, n, n_new)

    def fork(self, src: torch.Tensor, dst: torch.Tensor) -> torch.Tensor:
        """Sequences dst become copies of sequences src, on the same pages."""
        return bv.bv_pages_fork(self.table, self.lens, self.refs, self.page_size, src, dst)

    def compact(self) -> None:
        """The pages in use move to the front of the pools."""
        moves, count = bv.bv_pages_compact(self.table, self.lens, self.refs, self.page_size)
        for k, v in zip(self.k, self.v):
            bv.bv_pages_copy(k, v, moves, count)


class Decoder:
    """A decoder (workloads.attention_models) and its cache.  ``window`` and ``sinks`` as in bv_cache_attend."""

    def __init__(self, weights, B: int, capacity: int, page_size: int = 16, window: int = 0, sinks: int = 0):
        self.w, self.window, self.sinks = weights, window, sinks
        self.heads, self.kv_heads, self.D = weights["heads"], weights["kv_heads"], weights["head_dim"]
        e = weights["embed"]
        self.cache = PagedCache(len(weights["layers"]), B, capacity, self.kv_heads, self.D, page_size, e.dtype, e.device)

    def forward(self, tokens: torch.Tensor, lens: torch.Tensor, n_new=None) -> torch.Tensor:
        """Takes the newest tokens [B, n] (the cache has room for them; lens counts them in) through the layers; the logits
        [B, n, V] after each.  What is no token of the vocabulary (padding beyond n_new, a fault's -1) is taken for the nearest one."""
        c, B, n = self.cache, tokens.shape[0], tokens.shape[1]
        x = self.w["embed"][tokens.clamp(0, self.w["embed"].shape[0] - 1)]
        for layer, k, v in zip(self.w["layers"], c.k, c.v):
            qkv = (x @ layer["qkv"]).view(B, n, self.heads + 2 * self.kv_heads, self.D)
            q, kn, vn = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=2)
            bv.bv_cache_append(kn, vn, k, v, c.table, lens, n_new=n_new)
            o = bv.bv_cache_attend(q, k, v, c.table, lens, n_new=n_new, window=self.window, sinks=self.sinks)
            x = x + o.reshape(B, n, self.heads * self.D) @ layer["out"]
        return x @ self.w["unembed"]


def run(target: Decoder, draft: Decoder, prompts: torch.Tensor, prompt_lens: torch.Tensor, u_draft: torch.Tensor, u_verify: torch.Tensor,
        gamma: int, temperature: float = 1.0, algo: str = "block_lse", graph: bool = False) -> Dict[str, torch.Tensor]:
    """Run ``u_draft.shape[0]`` iterations of Algorithm 3 on two decoders with empty caches.

    prompts int32 [B, L] (CUDA), of which sequence b has prompt_lens[b] in 1 .. L (what lies beyond is not looked at); u_draft [N, gamma, B] and u_verify [N, B, gamma+2]: float32
    uniforms; algo as in ``specdec.run``.  Returns ``tokens`` int32 [B, N (gamma+1)] (generated tokens, then -1), ``lengths`` int64 [B], ``tau`` int32
    [N, B] and ``drafted`` int32 [N, B, gamma].  With ``graph`` the iterations after the first are replays of one captured one.
    """
    from .specdec import ALGOS
    if algo not in ALGOS:
        raise ValueError("algo must be one of %s" % (ALGOS,))
    N, B = u_draft.shape[0], prompts.shape[0]
    if prompts.dim() != 2 or prompts.dtype != torch.int32 or tuple(prompt_lens.shape) != (B,) or prompt_lens.dtype != torch.int32:
        raise ValueError("prompts must be int32 [B, L] and prompt_lens int32 [B]")
    if tuple(u_draft.shape) != (N, gamma, B) or tuple(u_verify.shape) != (N, B, gamma + 2):
        raise ValueError("u_draft must be [N, gamma, B] and u_verify [N, B, gamma+2]")
    # (one look of the host before anything is indexed by them: what is out of range would be a fault of the device)
    held = torch.arange(prompts.shape[1], device=prompts.device)[None, :] < prompt_lens[:, None]
    vocabulary = min(m.w["embed"].shape[0] for m in (target, draft))
    if bool(((prompt_lens < 1) | (prompt_lens > prompts.shape[1])).any() | (held & ((prompts < 0) | (prompts >= vocabulary))).any()):
        raise ValueError("prompt_lens must be in 1 .. %d, and tokens of the prompts in 0 .. %d" % (prompts.shape[1], vocabulary - 1))
    dev, width = prompts.device, N * (gamma + 1)
    V = target.w["unembed"].shape[1]
    fault = torch.zeros((1,), dtype=torch.int32, device=dev)
    # the prompts, but for their last tokens, which the first iteration takes in
    cur = prompts.gather(1, (prompt_lens - 1)[:, None].long()).squeeze(1)
    if prompts.shape[1] > 1:
        for m in (target, draft):
            new = m.cache.extend(prompts.shape[1] - 1, prompt_lens - 1)
            fault.add_((new < 0).any())
            m.forward(prompts[:, :-1], m.cache.lens, new)
    seq = torch.full((B, width + 1), -1, dtype=torch.int32, device=dev)
    pos = torch.zeros((B,), dtype=torch.int64, device=dev)
    taus = torch.empty((N, B), dtype=torch.int32, device=dev)
    drafted = torch.empty((N, B, gamma), dtype=torch.int32, device=dev)
    it = torch.zeros((1,), dtype=torch.int64, device=dev)          # the iteration number, on the device
    block = torch.empty((B, gamma + 1), dtype=torch.int32, device=dev)
    draft_logits = torch.empty((B, gamma, V), dtype=target.w["embed"].dtype, device=dev)
    lse = torch.empty((B, gamma), dtype=torch.float32, device=dev)
    col = torch.arange(gamma + 1, device=dev)
    step = torch.arange(1, gamma + 2, dtype=torch.int32, device=dev)[:, None]
    trash = torch.full((1,), width, dtype=torch.int64, device=dev)
    verify = {"block_lse": bv.bv_verify_lse, "token_lse": bv.tv_verify_lse, "block": bv.bv_verify, "token": bv.tv_verify}[algo]

    def iteration():
        ud, uv = u_draft.index_select(0, it)[0], u_verify.index_select(0, it)[0]
        at = draft.cache.lens + step                               # [gamma + 1, B]: lengths with 1, 2, ... tokens of the block
        for m in (target, draft):
            fault.add_((m.cache.extend(gamma + 1) < 0).any())
        block[:, 0] = cur
        # (the last drafted token goes through the draft model too: it is in the context if all of them are accepted)
        for i in range(gamma + 1):
            logits = draft.forward(block[:, i:i + 1], at[i])[:, 0]
            if i < gamma:
                draft_logits[:, i] = logits
                tok, row_lse = bv.bv_sample_draft(logits.contiguous(), ud[i], temperature)
                block[:, i + 1] = tok
                lse[:, i] = row_lse
        target_logits = target.forward(block, target.cache.lens).contiguous()
        toks = block[:, 1:].contiguous()
        given = (lse,) if algo.endswith("lse") else ()
        out, out_len = verify(target_logits, draft_logits, toks, uv.contiguous(), *given, temperature)
        for m in (target, draft):
            m.cache.truncate(out_len, gamma + 1)
        fault.add_((out_len < 1).any())
        n_out = out_len.to(torch.int64).clamp_(min=1)
        seq.scatter_(1, torch.where(col[None, :] < n_out[:, None], pos[:, None] + col[None, :], trash), out)
        cur.copy_(out.gather(1, (n_out - 1)[:, None]).squeeze(1))
        pos.add_(n_out)
        taus.index_copy_(0, it, (out_len - 1)[None, :])
        drafted.index_copy_(0, it, toks[None])
        it.add_(1)

    if graph and N > 1:
        # (the first iteration runs eagerly on the side stream: the library sizes that stream's workspace; the second is captured)
        side = torch.cuda.Stream(device=dev)
        side.wait_stream(torch.cuda.current_stream(dev))
        with torch.cuda.stream(side):
            iteration()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            iteration()
        torch.cuda.current_stream(dev).wait_stream(side)
        for _ in range(N - 1):
            g.replay()
    else:
        for _ in range(N):
            iteration()
    if int(fault.item()) != 0:
        raise RuntimeError("a sequence reported a data fault (out_len = -1), or a cache had no room for it")
    return dict(tokens=seq[:, :width].contiguous(), lengths=pos, tau=taus, drafted=drafted)
