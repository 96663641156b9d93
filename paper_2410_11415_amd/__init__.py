"""MI355X-native layered arithmetic-circuit evaluator (KLay hot path): HIP kernels behind a C ABI.

``binding`` holds the ctypes layer over ``lib/libklay.so``; ``build`` compiles it with hipcc; ``operators`` holds what stands between a
network and the leaf weights (log probabilities of tokens, from logits or straight from hidden states, distillation, gated recurrences),
``autograd`` the circuit as a layer.
"""
from .binding import (KLAY_AND, KLAY_FALSE, KLAY_LIT, KLAY_LOG, KLAY_MAXLOG, KLAY_OR, KLAY_REAL, KLAY_STATIC_WORKSPACE_BYTES, KLAY_TRUE,
                      Builder, Circuit, KlayError, klay_backward, klay_backward_f64, klay_backward_lits, klay_build, klay_destroy,
                      klay_forward, klay_distill_backward, klay_distill_forward, klay_forward_f64, klay_forward_lits, klay_forward_static,
                      klay_head_backward, klay_head_distill_backward, klay_head_distill_forward, klay_head_forward, klay_last_error,
                      klay_scan_backward, klay_scan_forward, klay_scan_step, klay_tokens_backward, klay_tokens_forward, library_path, load)

__all__ = ["KLAY_AND", "KLAY_FALSE", "KLAY_LIT", "KLAY_LOG", "KLAY_MAXLOG", "KLAY_OR", "KLAY_REAL", "KLAY_STATIC_WORKSPACE_BYTES",
           "KLAY_TRUE", "Builder", "Circuit", "KlayError", "klay_backward", "klay_backward_f64", "klay_backward_lits", "klay_build",
           "klay_destroy", "klay_distill_backward", "klay_distill_forward", "klay_forward", "klay_forward_f64", "klay_forward_lits",
           "klay_forward_static", "klay_head_backward", "klay_head_distill_backward", "klay_head_distill_forward", "klay_head_forward",
           "klay_last_error", "klay_scan_backward", "klay_scan_forward", "klay_scan_step", "klay_tokens_backward", "klay_tokens_forward",
           "library_path", "load"]


def __getattr__(name):
    # the torch layer is imported on first use, so that the binding alone does not need torch
    if name == "CircuitLayer":
        from .autograd import CircuitLayer
        return CircuitLayer
    if name in ("HeadLogprobs", "TokenLogprobs", "gated_scan", "gated_step", "head_distill", "head_logprobs", "token_distill", "token_logprobs"):
        from . import operators
        globals()[name] = getattr(operators, name)          # (found without this function from now on)
        return globals()[name]
    raise AttributeError(name)
