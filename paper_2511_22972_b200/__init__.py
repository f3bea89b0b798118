"""B200-native (sm_100a) FLy loose-verification step.

`binding` wraps the C ABI of libfly_verify.so (include/fly_verify.h);
`cache` wraps include/fly_cache.h (paged key/value cache, attention of a chunk over it);
`synthetic` draws the benchmark inputs; `build` compiles the library.
"""
from . import binding, build, cache, synthetic  # noqa: F401
from .binding import FlyError, FlyVerify, VerifyBuffers, verify, verify_fused  # noqa: F401
from .cache import ChunkAttention, PagedCache, cache_append, cache_read  # noqa: F401
