"""Decode-step GQA attention over ragged multi-turn KV caches on MI355X (gfx950),
with causal prefill of appended tokens, operators over paged caches, the fused OPD
token loss and token log probabilities with their gradient.

The kernels live in libctx_decode_attn.so (C ABI in include/ctx_decode_attn.h,
include/ctx_paged_attn.h, include/ctx_opd_loss.h and include/ctx_token_logprob.h);
`binding.DecodeAttention`, `binding.opd_loss` and `binding.token_logprobs` are the thin ctypes
wrappers used by tests and the benchmark.  Importing this package loads nothing; `workloads` holds
the seeded input generator.
"""

__all__ = ["AttnScores", "DecodeAttention", "CtxError", "OpdParams", "Rotary", "load_library", "opd_loss", "token_logprobs",
           "token_logprobs_grad"]


def __getattr__(name):
    if name in __all__:
        from . import binding

        value = globals()[name] = getattr(binding, name)  # found without this function from now on
        return value
    raise AttributeError(name)
