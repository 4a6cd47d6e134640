"""MI355X-native per-partition sampling + halo prefetch buffer + feature gather
(MassiveGNN, arXiv 2410.22697) behind the C ABI of include/massive.h.

`Massive` samples minibatches and gathers their rows; `operators` has what a
training step does with them: rows held in few bits (`RowFormat`, `pack_rows`,
`unpack_rows`), the mean over a sampled block (`block_mean`), a layer
(`linear`) and the step on the weights (`AdamW`). Everything runs in
libmassive's HIP kernels; making a `Massive`, or calling an operator, raises
if libmassive.so has not been built.
"""
from .massive import (EXPORTS, LIB_PATH, MAX_INFLIGHT, TIMING_GROUPS, BatchBuffers, Massive,  # noqa: F401
                      MassiveError, StepResult, load)
from .operators import (AdamW, RowFormat, block_mean, block_mean_backward, linear, linear_backward,  # noqa: F401
                        pack_rows, unpack_rows)
