"""streambeam: streaming variable-width batched beam search on MI355X (gfx950).

The search step of Var-Stream (Yang et al., EMNLP 2020, Sec. 3 / Alg. 1) and
its settings Fixed and Var-Batch, as hand-written HIP kernels behind a C ABI
(include/streambeam.h), and the operators of a serving step for cached
transformer decoders next to it (serving.py). This package holds the ctypes
binding and the build script; PyTorch only provides device memory and streams.
"""
from .decoder import (Decoder, Hypothesis, decoder_for_workload, group_by_input, inputs_to_device,
                      weights_to_device)

_SERVING = ("PagePlan", "int8_linear", "page_bounds", "paged_attention", "plan_pages", "quantize_rows", "rope_append",
            "rope_frequencies", "sample_tokens", "select_pages", "selected_attention", "shared_attention")

__all__ = ["Decoder", "Hypothesis", "decoder_for_workload", "group_by_input", "inputs_to_device",
           "weights_to_device", *_SERVING]


def __getattr__(name):
    # serving.py needs torch from the start, the rest only with a GPU at hand.
    if name in _SERVING:
        from . import serving
        globals().update({n: getattr(serving, n) for n in _SERVING})
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
