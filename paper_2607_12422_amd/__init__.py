"""MI355X-native PEFT-BD speculative step: HIP kernels behind a C ABI (libpbd).

``binding`` marshals arguments to the library (the product path); ``costmodel``
holds the paper's host-side cost arithmetic used for reporting; ``build``
compiles the library in-tree for gfx950.
"""
from . import binding, costmodel  # noqa: F401
from .binding import (Engine, load_library, make_config, make_pages, pbd_paged_append, pbd_paged_attention,  # noqa: F401
                      pbd_paged_evict, pbd_token_logprobs, upload_weights)
