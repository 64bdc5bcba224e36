"""ARCHead packed LM-head forward for AMD Instinct MI355X (gfx950).

The compute path is the C-ABI library libarchead.so (hand-written HIP
kernels); ``archead`` is its thin ctypes binding, with PyTorch providing
device memory and streams only.
"""
from .archead import (  # noqa: F401
    ArcheadError,
    BeamStates,
    BuildDesc,
    Desc,
    beam_select,
    build_head,
    PackedHead,
    logit_fidelity,
    lib,
    matmul_i8,
    pack_int4,
    pack_int5,
    packed_bytes,
    quantize_i8,
    unpack_int4,
    unpack_int5,
    validate_desc,
)
