"""CollectiveKV for NVIDIA B200: a C-ABI CUDA library (libckv.so, declared in include/ckv.h) and this thin Python binding.
It holds the decode-stage hot path, the prefill router and projection, and the calls of a training step that fit the router and
the pool.  PyTorch is used by callers only for device memory and streams."""
from .binding import *  # noqa: F401,F403
from .binding import CkvError, EXPORTS, LIB_PATH, lib  # noqa: F401
from .session import CollectiveKV  # noqa: F401
from .fit import gather, gather_grad, route_loss, route_loss_grad, sort_indices  # noqa: F401
