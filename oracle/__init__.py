"""CPU oracle for the Distance-KV hot path (test infrastructure only).

Only the tests, the package smoke check and the benchmark's CPU-baseline leg
may import this package.  See `dkv_oracle` for what it computes, and
`page_fill` for paged caches that are filled on the GPU, and `tree_cache` for
rotary positions, quantised rows and drafted trees.
"""

from . import page_fill, tree_cache  # noqa: F401
from .dkv_oracle import *  # noqa: F401,F403
from .dkv_oracle import __all__  # noqa: F401
