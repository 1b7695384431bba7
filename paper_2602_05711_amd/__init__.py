"""MI355X (gfx950) implementation of the OmniMoE atomic-expert layer forward pass.

The computation lives in libomnimoe.so (HIP kernels behind the C ABI of include/);
``binding`` exposes the same entry points to Python for torch tensors.
"""
from .binding import (  # noqa: F401
    EXPORTED, EXPORTED_BLOCK, EXPORTED_FFN, FEW_TOKENS, KERNEL_NAMES, ORDERS, OmnimoeAdapters, OmnimoeError,
    OmnimoeLayerDesc, OmnimoeProduct, Timer,
    load_library, make_adapters, make_desc, make_product,
    omnimoe_block_join, omnimoe_block_join_backward, omnimoe_block_join_backward_workspace_size,
    omnimoe_checkpoint_load, omnimoe_checkpoint_store,
    omnimoe_expert_backward, omnimoe_expert_forward, omnimoe_expert_forward_grouped,
    omnimoe_expert_forward_group_rows, omnimoe_expert_forward_scatter,
    omnimoe_expert_forward_token_centric,
    omnimoe_grouped_product, omnimoe_grouped_product4, omnimoe_grouped_product_dw,
    omnimoe_grouped_product_dw_workspace_size, omnimoe_grouped_product_dx,
    omnimoe_layer_few_workspace_size, omnimoe_layer_forward, omnimoe_layer_forward_few,
    omnimoe_layer_forward_noalloc, omnimoe_layer_kernels, omnimoe_layer_path,
    omnimoe_route, omnimoe_route_backward, omnimoe_route_dense, omnimoe_schedule, omnimoe_select, omnimoe_select_dense,
    omnimoe_shared_mlp, omnimoe_shared_mlp_adapters, omnimoe_shared_mlp_adapters_workspace_size,
    omnimoe_shared_mlp_backward, omnimoe_shared_mlp_backward_workspace_size,
    omnimoe_shared_mlp_workspace_size, omnimoe_weights4_load, omnimoe_weights4_store,
    omnimoe_workspace_size, workspace,
)
