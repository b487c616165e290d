"""Per-GPU rehearsal buffer for MI355X (gfx950): C-ABI HIP library plus a thin binding (ctypes, native for most calls of a training loop).

Importing this package loads paper_2406_03285_amd/librb.so (the buffer), librb_train.so (the operators of the training step it feeds) and
librb_block.so (what a model's blocks compute between their matrix products) and fails if they have not been built (`python paper_2406_03285_amd/build.py`); there is no CPU path.
"""
from .binding import *  # noqa: F401,F403
from .binding import RehearsalBuffer, Pipeline, RbError, EXPORTS, LIB_PATH  # noqa: F401
from .train import *  # noqa: F401,F403
from .block import *  # noqa: F401,F403
