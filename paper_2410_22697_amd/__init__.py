"""MI355X-native per-partition sampling + halo prefetch buffer + feature gather
(MassiveGNN, arXiv 2410.22697) behind the C ABI of include/massive.h.

`Massive` samples minibatches and gathers their rows; `operators` has what a
training step does with them: rows held in few bits (`RowFormat`, `pack_rows`,
`unpack_rows`), the mean over a sampled block (`block_mean`), a layer
(`linear`), a gated one (`gated`), the norm and the dropout between them
(`rms_norm`, `dropout`) and the step on the weights (`AdamW`). Everything runs
in libmassive's HIP kernels; making a `Massive`, or calling an operator, raises
if libmassive.so has not been built.
"""
import importlib

from .massive import (EXPORTS, LIB_PATH, MAX_INFLIGHT, TIMING_GROUPS, BatchBuffers, Massive,  # noqa: F401
                      MassiveError, StepResult, load)

# what needs torch is loaded when it is first asked for
_OPERATORS = ("AdamW", "RowFormat", "block_mean", "block_mean_backward", "dropout", "dropout_backward", "gated", "gated_backward", "linear", "linear_backward", "pack_rows",
              "rms_norm", "rms_norm_backward", "unpack_rows")
__all__ = ["EXPORTS", "LIB_PATH", "MAX_INFLIGHT", "TIMING_GROUPS", "BatchBuffers", "Massive", "MassiveError", "StepResult", "load", "massive",
           "operators", *_OPERATORS]


def __getattr__(name):
    if name not in _OPERATORS and name != "operators":
        raise AttributeError("module %r has no attribute %r" % (__name__, name))
    operators = importlib.import_module(".operators", __name__)
    globals().update({n: getattr(operators, n) for n in _OPERATORS})
    return operators if name == "operators" else globals()[name]


def __dir__():
    return sorted([*globals(), "operators", *_OPERATORS])
