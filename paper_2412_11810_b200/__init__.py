"""B200 (sm_100a) BPTT training step for sparse recurrent / spiking networks under the
gradient-checkpointing strategies of arXiv 2412.11810.  The CUDA library sits behind the C ABI
of include/snn.h; `binding` mirrors it, `session` owns the torch buffers and streams, `ops` are the sequence-model
operators (gated linear recurrence, 8-bit activations, vocabulary loss) on torch tensors."""
from . import binding  # noqa: F401  (fails loudly if the CUDA library is missing)
from . import ops  # noqa: F401
from .session import Session  # noqa: F401
