"""From a prompt to a verified block, through the C ABI.

A verification step (step.py) starts from a cache that already holds the
prefix and from drafts.  This module is the way there:

  1. simsd_rope_append     a prompt chunk's q rotated, its keys (rotated) and
     values written to the pages, per layer
  2. simsd_chunk_attention the chunk's attention over all that is cached
  3. simsd_sample          drafts from the draft model's logits, with the
     truncated distribution they were drawn from; the same truncation of the
     target's logits
  4. simsd_build_mask, simsd_rope_rotate, simsd_verify_attention per layer
  5. simsd_accept_sampled  Eq. (2) on the two truncated distributions
  6. simsd_kv_commit       the accepted drafts' keys and values

Long contexts: the cache may be held in 4 bits (simsd_rope_append_q4 and
simsd_chunk_attention_q4 in place of calls 1 and 2), attention may go through
a window beside which the first rows stay visible
(simsd_chunk_attention_sinks), and the pages may come from a pool that is
smaller than all sequences together: simsd_pages_extend before a chunk,
simsd_pages_release of what the window has left behind, simsd_pages_fork for
several continuations of one prompt, simsd_pages_compact.

The rotation may be one that the verification kernels do not do themselves
(interleaved, partial or scaled for long contexts): q and the new keys are
rotated by simsd_rope_rotate at the RoPE-copy positions first (Sec. 3.1).
``python -m paper_2606_02544_gb300.prompt`` runs all of it on random tensors.
"""
from __future__ import annotations

import torch

from . import simsd


class PromptCache:
    """The paged cache of ``layers`` attention layers and the calls that fill
    and read it.  PyTorch only allocates the buffers."""

    def __init__(self, layers, Bt, Hq, Hkv, d, page_size, max_len, plan, mask_block=1, dtype=torch.bfloat16,
                 device="cuda", window=0, sinks=0, bits=None, pages=None):
        """window, sinks: rows back, and first rows, that a token sees (0: all);
        bits 4: the cache in 4 bits; pages: size of a pool whose pages the
        sequences take and let go of (None: a place for every row)."""
        if bits not in (None, 4) or window < 0 or sinks < 0:
            raise ValueError("bits: None or 4; window and sinks: 0 or more")
        self.L, self.Bt, self.Hq, self.Hkv, self.d, self.P = layers, Bt, Hq, Hkv, d, page_size
        self.plan, self.mask_block, self.dtype, self.device = plan, mask_block, dtype, device
        self.window, self.sinks, self.bits, self.pooled = window, sinks, bits, pages is not None
        self.code = simsd.SIMSD_F32 if dtype == torch.float32 else simsd.SIMSD_BF16
        self.max_pages = (max_len + page_size - 1) // page_size
        pages = Bt * self.max_pages if pages is None else pages
        i32 = dict(dtype=torch.int32, device=device)
        if bits == 4:
            parts = [torch.zeros(layers, pages, Hkv, page_size, w, dtype=torch.uint8, device=device)
                     for w in (d // 2, d // 16) * 2]
            self.q4 = [simsd.Q4Cache(*(x[l] for x in parts)) for l in range(layers)]
        else:
            self.k_cache = torch.empty(layers, pages, Hkv, page_size, d, dtype=dtype, device=device)
            self.v_cache = torch.empty_like(self.k_cache)
            parts = [self.k_cache, self.v_cache]
        if self.pooled:
            self.page_set = simsd.PageSet(parts)
            self.block_table = torch.full((Bt, self.max_pages), -1, **i32)
        else:
            self.block_table = torch.arange(pages, **i32).view(Bt, self.max_pages)
        self.refs = torch.zeros(pages, **i32)
        self.live = torch.zeros(1, **i32)
        self.prefix_len = torch.zeros(Bt, **i32)
        self.err = torch.zeros(1, **i32)
        self.workspace, self.captured = None, []

    def _scratch(self, nbytes):
        if nbytes and (self.workspace is None or self.workspace.numel() < nbytes):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        if not nbytes:
            return None
        # a graph goes on writing to the workspace it was captured with: it is kept
        if torch.cuda.is_current_stream_capturing() and not any(w is self.workspace for w in self.captured):
            self.captured.append(self.workspace)
        return self.workspace

    def _pool(self):
        if not self.pooled:
            raise ValueError("a cache with a place for every row has no pool: make it with pages")

    def append_chunk(self, qkv, token_start):
        """One chunk of every layer: qkv [L][T][Hq + 2 Hkv][d] (rows of the
        layers' projections), token_start [Bt+1].  Returns the attention
        outputs [L][T][Hq][d] and advances the prefix lengths.

        With a pool, sequences that get no pages (too few are free:
        SIMSD_EW_POOL in err, and those that want none go on; or they would
        write to a page that another one shares, having been cut back:
        SIMSD_EW_SHARED; SIMSD_EW_PREFIX_LEN besides) stay as they were:
        length, pages and rows, with outputs of zero.  Their rows can be given
        again once pages are free."""
        T = qkv.shape[1]
        Hq, Hkv = self.Hq, self.Hkv
        lengths = token_start[1:] - token_start[:-1]
        lens = self.prefix_len
        if self.pooled:
            lens = torch.empty_like(lens)  # -1: a sequence that is not to be written
            simsd.simsd_pages_extend(self.prefix_len, lengths, self.block_table, self.refs, self.P, err_word=self.err,
                                     granted=lens)
        out = torch.empty(self.L, T, Hq, self.d, dtype=self.dtype, device=self.device)
        q = torch.empty(T, Hq, self.d, dtype=self.dtype, device=self.device)
        sizes = (self.code, T, self.Bt, Hq, Hkv, self.d, self.max_pages, self.P)
        ws = self._scratch(simsd.simsd_chunk_q4_workspace_bytes(*sizes, self.refs.shape[0]) if self.bits == 4
                           else simsd.simsd_chunk_workspace_bytes(*sizes))
        for l in range(self.L):
            x = qkv[l]
            args = (self.plan, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], token_start, lens, q)
            if self.bits == 4:
                simsd.simsd_rope_append_q4(*args, self.q4[l], self.block_table, err_word=self.err)
                simsd.simsd_chunk_attention_q4(q, token_start, lens, self.q4[l], self.block_table, out[l],
                                               mask_block=self.mask_block, window=self.window, sinks=self.sinks,
                                               workspace=ws, err_word=self.err)
                continue
            cache = (self.k_cache[l], self.v_cache[l], self.block_table)
            simsd.simsd_rope_append(*args, *cache, err_word=self.err)
            if self.window:
                simsd.simsd_chunk_attention_sinks(q, token_start, lens, *cache, out[l], self.window,
                                                  self.sinks, mask_block=self.mask_block, workspace=ws,
                                                  err_word=self.err)
            else:
                simsd.simsd_chunk_attention(q, token_start, lens, *cache, out[l],
                                            mask_block=self.mask_block, workspace=ws, err_word=self.err)
        self.prefix_len += lengths.masked_fill(lens < 0, 0) if self.pooled else lengths
        if self.pooled and self.window:
            # the next token sees rows from prefix_len + 1 - window on, and the first ones
            first = torch.full_like(self.prefix_len, self.sinks)
            simsd.simsd_pages_release(self.block_table, self.refs, first, self.prefix_len + (1 - self.window), self.P,
                                      err_word=self.err)
        return out

    def fork(self, src, dst):
        """Sequences dst become copies of sequences src (int32 tensors)."""
        self._pool()
        ws = self._scratch(simsd.simsd_pages_workspace_bytes(0, src.shape[0]))
        simsd.simsd_pages_fork(self.page_set, src, dst, self.prefix_len, self.block_table, self.refs, self.P,
                               workspace=ws, err_word=self.err)

    def release(self, seq):
        """Sequences seq (an int32 tensor) end."""
        self._pool()
        zero = torch.zeros_like(seq)
        simsd.simsd_pages_release(self.block_table, self.refs, zero, torch.full_like(seq, 2 ** 31 - 1), self.P,
                                  seq=seq, err_word=self.err)
        # (a number out of range, which sets SIMSD_EW_SEQ, is none of the rows)
        rows = torch.arange(self.Bt, dtype=torch.int32, device=self.device)
        self.prefix_len.masked_fill_((rows[:, None] == seq).any(1), 0)

    def compact(self):
        """Moves the pages in use to the lowest ids; their number, on the GPU."""
        self._pool()
        ws = self._scratch(simsd.simsd_pages_workspace_bytes(self.refs.shape[0]))
        simsd.simsd_pages_compact(self.page_set, self.block_table, self.refs, self.live, workspace=ws,
                                  err_word=self.err)
        return self.live

    def draw(self, logits, u, **limits):
        """Tokens of logits [..][V] under random numbers u [..], and the
        log-probabilities of the truncated distribution they come from."""
        V = logits.shape[-1]
        rows = logits.reshape(-1, V)
        token = torch.empty(rows.shape[0], dtype=torch.int32, device=self.device)
        log_probs = torch.empty(rows.shape, dtype=torch.float32, device=self.device)
        simsd.simsd_sample(rows, u.reshape(-1), token, log_probs=log_probs, err_word=self.err, **limits)
        return token.view(logits.shape[:-1]), log_probs.view(logits.shape)

    def verify(self, q, k_new, v_new, draft, target_log_probs, draft_log_probs, u_accept, u_sample):
        """One verification step on drafts with their distributions: q
        [L][Bt][2g][Hq][d], k_new / v_new [L][Bt][2g][Hkv][d] not rotated (they
        are rotated in place), target_log_probs [Bt][g+1][V], draft_log_probs
        [Bt][g][V].  Returns outputs, accepted lengths and tokens.  The prefix is
        read whole, from a cache in dtype (simsd_q4_expand makes one of a cache
        in 4 bits)."""
        if self.bits == 4 or self.window or self.pooled:
            raise ValueError("verification reads a whole cache in its own type, with a place for every row")
        L, Bt, S, Hq, d = q.shape
        gamma = S // 2
        i32 = dict(dtype=torch.int32, device=self.device)
        tau, rope_pos = torch.empty(Bt, S, **i32), torch.empty(Bt, S, **i32)
        section = torch.empty(Bt, S, dtype=torch.uint8, device=self.device)
        simsd.simsd_build_mask(None, self.prefix_len, gamma, tau, section, rope_pos, err_word=self.err)
        ws = self._scratch(simsd.simsd_verify_workspace_bytes(self.code, Bt, gamma, Hq, self.Hkv, d, self.max_pages,
                                                              self.P))
        out = torch.empty_like(q)
        for l in range(L):
            ql, kl = q[l].view(-1, Hq, d), k_new[l].view(-1, self.Hkv, d)
            simsd.simsd_rope_rotate(self.plan, rope_pos.view(-1), ql, ql, kl, kl)
            simsd.simsd_verify_attention(q[l], k_new[l], v_new[l], self.k_cache[l], self.v_cache[l],
                                         self.block_table, self.prefix_len, tau, section, out[l], workspace=ws,
                                         err_word=self.err)
        accepted, tokens = torch.empty(Bt, **i32), torch.empty(Bt, gamma + 1, **i32)
        simsd.simsd_accept_sampled(target_log_probs, draft_log_probs, draft, u_accept, u_sample, accepted, tokens,
                                   err_word=self.err)
        simsd.simsd_kv_commit(k_new, v_new, tau, section, accepted, self.k_cache, self.v_cache, self.block_table,
                              self.prefix_len, err_word=self.err)
        return out, accepted, tokens


def main():
    """Prompts of odd lengths in chunks, then one verified block."""
    g = torch.Generator(device="cuda").manual_seed(0)
    layers, Bt, Hq, Hkv, d, gamma, V = 4, 4, 16, 8, 128, 8, 151936
    plan = simsd.simsd_rope_plan_init("half", d, 1.0e6, "yarn", factor=4.0, context=8192)
    cache = PromptCache(layers, Bt, Hq, Hkv, d, 64, 4096, plan, mask_block=gamma)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    lengths, step, done = [1203, 77, 2040, 512], 512, [0] * Bt
    while any(a < b for a, b in zip(done, lengths)):
        chunk = [min(step, b - a) for a, b in zip(done, lengths)]
        start = torch.tensor([sum(chunk[:i]) for i in range(Bt + 1)], dtype=torch.int32, device="cuda")
        cache.append_chunk((randn(layers, sum(chunk), Hq + 2 * Hkv, d) * d ** -0.25).bfloat16(), start)
        done = [a + c for a, c in zip(done, chunk)]
    target = randn(Bt, gamma + 1, V) * 3.0
    limits = lambda n: dict(  # noqa: E731
        temperature=torch.full((n,), 0.8, device="cuda"), top_p=torch.full((n,), 0.95, device="cuda"),
        top_k=torch.full((n,), 50, dtype=torch.int32, device="cuda"))
    draft, draft_lp = cache.draw(target[:, :gamma] + 0.3 * randn(Bt, gamma, V), rand(Bt, gamma), **limits(Bt * gamma))
    _, target_lp = cache.draw(target, rand(Bt, gamma + 1), **limits(Bt * (gamma + 1)))
    new = lambda h: (randn(layers, Bt, 2 * gamma, h, d) * d ** -0.25).bfloat16()  # noqa: E731
    out, accepted, tokens = cache.verify(new(Hq), new(Hkv), new(Hkv), draft, target_lp, draft_lp, rand(Bt, gamma),
                                         rand(Bt))
    word = simsd.simsd_check_error(cache.err)
    print(f"prompts {lengths}, accepted {accepted.tolist()} of {gamma}, cached {cache.prefix_len.tolist()}, "
          f"error word {word}")
    print("tokens", tokens.tolist())
    fine = long_context(plan)
    return 0 if fine and word == 0 and bool(torch.isfinite(out.float()).all()) else 1


def long_context(plan):
    """One prompt, four continuations through a window over a cache in 4 bits,
    in a pool of a few pages."""
    g = torch.Generator(device="cuda").manual_seed(1)
    layers, Hq, Hkv, d, i32 = 2, 16, 8, 128, dict(dtype=torch.int32, device="cuda")
    cache = PromptCache(layers, 4, Hq, Hkv, d, 64, 65536, plan, window=1024, sinks=64, bits=4, pages=100)
    chunk = lambda *n: (  # noqa: E731
        (torch.randn(layers, sum(n), Hq + 2 * Hkv, d, generator=g, device="cuda") * d ** -0.25).bfloat16(),
        torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], **i32))
    for _ in range(6):
        out = cache.append_chunk(*chunk(1000, 0, 0, 0))
    cache.fork(torch.zeros(3, **i32), torch.arange(1, 4, **i32))
    for _ in range(20):
        out = cache.append_chunk(*chunk(1, 1, 1, 1))
    cache.release(torch.tensor([0, 2], **i32))
    live = cache.compact()
    out = cache.append_chunk(*chunk(0, 1, 0, 1))
    word = simsd.simsd_check_error(cache.err)
    print(f"continuations at {cache.prefix_len.tolist()}, {int(live)} of 100 pages in use, error word {word}")
    return word == 0 and bool(torch.isfinite(out.float()).all())


if __name__ == "__main__":
    raise SystemExit(main())
