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
                 device="cuda"):
        self.L, self.Bt, self.Hq, self.Hkv, self.d, self.P = layers, Bt, Hq, Hkv, d, page_size
        self.plan, self.mask_block, self.dtype, self.device = plan, mask_block, dtype, device
        self.code = simsd.SIMSD_F32 if dtype == torch.float32 else simsd.SIMSD_BF16
        self.max_pages = (max_len + page_size - 1) // page_size
        pages = Bt * self.max_pages
        i32 = dict(dtype=torch.int32, device=device)
        self.k_cache = torch.empty(layers, pages, Hkv, page_size, d, dtype=dtype, device=device)
        self.v_cache = torch.empty_like(self.k_cache)
        self.block_table = torch.arange(pages, **i32).view(Bt, self.max_pages)
        self.prefix_len = torch.zeros(Bt, **i32)
        self.err = torch.zeros(1, **i32)
        self.workspace = None

    def _scratch(self, nbytes):
        if nbytes and (self.workspace is None or self.workspace.numel() < nbytes):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return self.workspace if nbytes else None

    def append_chunk(self, qkv, token_start):
        """One chunk of every layer: qkv [L][T][Hq + 2 Hkv][d] (rows of the
        layers' projections), token_start [Bt+1].  Returns the attention
        outputs [L][T][Hq][d] and advances the prefix lengths."""
        T = qkv.shape[1]
        Hq, Hkv = self.Hq, self.Hkv
        out = torch.empty(self.L, T, Hq, self.d, dtype=self.dtype, device=self.device)
        q = torch.empty(T, Hq, self.d, dtype=self.dtype, device=self.device)
        ws = self._scratch(simsd.simsd_chunk_workspace_bytes(self.code, T, self.Bt, Hq, Hkv, self.d, self.max_pages,
                                                             self.P))
        for l in range(self.L):
            x = qkv[l]
            simsd.simsd_rope_append(self.plan, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], token_start,
                                    self.prefix_len, q, self.k_cache[l], self.v_cache[l], self.block_table,
                                    err_word=self.err)
            simsd.simsd_chunk_attention(q, token_start, self.prefix_len, self.k_cache[l], self.v_cache[l],
                                        self.block_table, out[l], mask_block=self.mask_block, workspace=ws,
                                        err_word=self.err)
        self.prefix_len += token_start[1:] - token_start[:-1]
        return out

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
        [Bt][g][V].  Returns outputs, accepted lengths and tokens."""
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
    return 0 if word == 0 and bool(torch.isfinite(out.float()).all()) else 1


if __name__ == "__main__":
    raise SystemExit(main())
