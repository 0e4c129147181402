"""B200 (sm_100a) Amphista speculative-decoding step: ctypes binding of libamph.so."""
from .binding import (  # noqa: F401
    Adapters,
    AmphError,
    Amphista,
    PagedCache,
    amph_config,
    amph_tensor,
    amph_tree,
    lib,
    library_path,
    make_config,
    make_tree,
    paged_attention,
    paged_write,
    project,
    project_adapters,
    project_noalloc,
)
