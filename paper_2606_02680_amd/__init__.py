"""MI355X-native Post-Boundary Bridge (PBB) decode attention.

The product is ``libpbb.so`` (C ABI in ``include/pbb.h``, HIP kernels for gfx950 in
``csrc/``); :mod:`paper_2606_02680_amd.pbb` is its thin ctypes binding.
"""
from .pbb import (  # noqa: F401
    PbbDesc, PbbError, PbbNorm, PbbPagedDesc, PbbRope, alloc_norm_workspace, alloc_coded_workspace,
    alloc_paged_workspace, alloc_pages, alloc_coded_pages, alloc_rings, alloc_workspace,
    backward_workspace_bytes, load_library, make_desc, make_paged_desc, make_rope, norm_workspace_bytes,
    coded_workspace_bytes, paged_workspace_bytes, pages_shape, pbb_backward, pbb_decode_step,
    pbb_decode_step_advance, pbb_decode_step_noalloc, pbb_norm_rotate, pbb_norm_rotate_backward,
    pbb_coded_append, pbb_coded_attention, pbb_coded_read, pbb_paged_append, pbb_paged_attention,
    pbb_prefill, pbb_rotate, ring_bytes, ring_fill, ring_init, ring_shape, scales_shape, swa_backward,
    swa_decode_step, swa_decode_step_advance, swa_prefill, swa_workspace_bytes, workspace_bytes)
