"""MI355X-native on-GPU decompression of the Endor bitmap sparse format.

`binding` is the thin ctypes layer over the C-ABI library (include/endor.h);
`decode` is the same for the decode side (paged key-value cache, attention,
eviction, 4-bit products);
`synth` draws the seeded synthetic pruned matrices used as inputs.
"""
from . import binding, decode, synth  # noqa: F401
from .binding import *  # noqa: F401,F403
from .decode import *  # noqa: F401,F403
