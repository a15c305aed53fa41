"""MI355X-native BitStack linear layer: thin ctypes binding over libbitstack.so.

Every step of the forward pass runs inside the HIP library; this package only
marshals arguments.  PyTorch supplies device memory and streams.
"""
from .binding import (  # noqa: F401
    BitStackError,
    PackedStack,
    BlockManager,
    TokenPlan,
    order_check,
    budget_position,
    KERNEL_AUTO, KERNEL_REFERENCE, KERNEL_DECODE, KERNEL_PANEL, KERNEL_MATERIALISE,
    OPT_DECODE_BGROUPS, OPT_DECODE_TILES, OPT_DECODE_KS_CHUNKS, OPT_DECODE_EARLY, OPT_DENSE_TILE, OPT_BATCH_TILES, OPT_ROWS_CHUNKS, OPT_F8_KERNEL,
    block_bytes,
    block_staging_bytes,
    dense_bytes,
    decompose,
    choose_kernel,
    restore_max_blocks,
    stage_block_host,
    lib,
    linear_many,
    make_jobs,
    lib_path,
    pack_image_host,
    pack_signs_from_f32,
    packed_bytes,
    probe_read,
    set_option,
    strerror,
    unpack_image_host,
)

_F8 = ("F8Rows", "Routing", "combine", "expert_layer_f8", "expert_layer_workspace_bytes", "f8_epilogue_workspace_bytes", "f8_workspace_bytes", "grouped_linear_f8", "linear_f8", "quantise_f8", "quantise_weight_f8", "route")


def __getattr__(name):
    """The 8-bit products and the routing (f8.py) need PyTorch: loaded at their first use."""
    if name not in _F8:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from . import f8
    globals().update({n: getattr(f8, n) for n in _F8})
    return globals()[name]
