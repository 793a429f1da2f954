"""CacheRepair repair forward pass on MI355X (gfx950).

The product is the HIP C-ABI library ``libcacherepair.so`` (declared in
``include/cacherepair.h``).  ``binding`` is its thin ctypes binding with the
same function names; ``repairer.Repairer`` adds torch device-buffer
marshalling, ``serving.PagedCache`` answers over a paged cache and
``serving.sample`` draws tokens.  There is
no CPU or fallback implementation: if the library is not built, loading it
raises.
"""
from .binding import (  # noqa: F401
    CR_DTYPE_BF16, CR_DTYPE_F32, CrError, cr_append_kv, cr_attend, cr_attend_workspace_bytes,
    cr_choose_slots, cr_chunk_schedule, cr_compact_kv, cr_dims, cr_kv_layout, cr_prepare_weights,
    cr_prepared_bytes, cr_repair, cr_sample, cr_status_string, cr_version, cr_weigh_keys,
    cr_weigh_workspace_bytes, cr_weights_layout, cr_workspace_bytes, cr_workspace_view,
    layer_major_layout, load,
    make_dims,
)


def __getattr__(name):
    if name == "Repairer":
        from .repairer import Repairer
        return Repairer
    if name == "PagedCache":
        from .serving import PagedCache
        return PagedCache
    if name == "sample":
        from .serving import sample
        return sample
    raise AttributeError(name)
