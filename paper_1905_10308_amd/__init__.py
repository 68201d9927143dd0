"""SCRAM hot path on MI355X: PatchMatch argmax + sparse window attention.

The computation lives in the HIP library ``_lib/libscram.so`` (C ABI:
``include/scram.h``); this package only marshals torch tensors into it.
Importing the package does not load the library; the first call does, and
raises if it is missing.
"""
from .binding import (  # noqa: F401
    CAUSAL,
    MAX_KAPPA,
    MAX_PREV,
    NOALLOC_MAX_QUERIES,
    NO_PROPAGATION,
    NO_RANDOM_SEARCH,
    ScramError,
    forward,
    lib,
    patchmatch,
    patchmatch_kappa,
    patchmatch_noalloc,
    patchmatch_workspace_bytes,
    snis_attend,
    sparse_attend,
    sparse_attend_backward,
    sparse_attend_backward_workspace_bytes,
    status_string,
)
from .dense import (  # noqa: F401
    bias_edges,
    dense_attend,
    dense_attend_backward,
    dense_attend_backward_workspace_bytes,
    dense_attend_workspace_bytes,
    relative_bias,
    relative_bias_backward,
    relative_bias_backward_workspace_bytes,
)
from .differential import (  # noqa: F401
    differential_attend,
    differential_attend_backward,
    differential_attend_backward_workspace_bytes,
)
from .rows import (  # noqa: F401
    group_norm,
    group_norm_backward,
    group_norm_backward_workspace_bytes,
    group_norm_workspace_bytes,
    layer_norm,
    layer_norm_backward,
    layer_norm_backward_workspace_bytes,
    rotary,
    rotary_backward,
)
