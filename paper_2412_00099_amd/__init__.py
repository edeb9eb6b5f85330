"""MI355X (gfx950) batch-1 MoE decode with cache-conditional routing: Python binding of libmoe_cache.

Importing the package loads the HIP library; there is no CPU fallback.  If the library has not been
built the import raises, naming the build command.  The operators on many rows and attention for tensors are a module
of their own: where only that one is missing, their names raise when they are used.
"""
from .binding import *  # noqa: F401,F403
from .binding import LIB_PATH, lib  # noqa: F401
from .runtime import ExpertStore, MoEDecoder  # noqa: F401
try:
    from .rows import (  # noqa: F401
        KeptExperts, NormedRows, TokenOrder, combine_rows, combine_rows_backward, experts_rows, experts_rows_backward, gather_rows,
        norm_rows, norm_rows_backward, sort_tokens,
    )
    from .attention import (  # noqa: F401
        KeptAttention, PagePlan, attend_pages, attend_rows, attend_rows_backward, plan_pages, store_pages,
    )
except ImportError as e:
    _rows_missing = str(e)

    def __getattr__(name):
        if name in ("rows", "KeptExperts", "NormedRows", "TokenOrder", "combine_rows", "combine_rows_backward", "experts_rows",
                    "experts_rows_backward", "gather_rows", "norm_rows", "norm_rows_backward", "sort_tokens",
                    "attention", "KeptAttention", "PagePlan", "attend_pages", "attend_rows", "attend_rows_backward", "plan_pages", "store_pages"):
            raise ImportError(_rows_missing)
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
