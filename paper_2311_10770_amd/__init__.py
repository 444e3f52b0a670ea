"""MI355X-native fast-feedforward (FFF) inference: conditional matrix multiplication on gfx950.

The compute lives in ``libfff.so`` (HIP kernels behind the C ABI of
``include/fff.h``); this package is its ctypes binding plus the seeded
synthetic-input generators and the named workloads.  ``ops`` holds the operators
around the layer: LayerNorm and dropout with their gradients, and the leaf
experts' grouped products; ``routed`` those of a routed expert block: routing, the sum of
a token's experts, RMS norm and activations kept in 8 bits.
"""
from .fff import (  # noqa: F401
    FffArgs, FffBackwardArgs, FffError, FffLayer, backward, backward_workspace_bytes, describe, describe_stack,
    forward, forward_plain, forward_stack, forward_static, from_numpy, load_library, make_args, status_str, to_numpy, version,
    workspace_bytes,
)
from .ops import (  # noqa: F401
    describe_grouped_matmul, describe_grouped_weight_grad, dropout, group_rows, group_rows_workspace_bytes,
    grouped_matmul, grouped_weight_grad, grouped_weight_grad_workspace_bytes, layer_norm, layer_norm_backward,
    layer_norm_backward_workspace_bytes,
)
from .routed import (  # noqa: F401
    Packed, activation_backward, combine, combine_backward, pack_rows, rms_norm, rms_norm_backward,
    rms_norm_backward_workspace_bytes, route, route_backward, unpack_rows,
)
