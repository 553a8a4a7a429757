"""MI355X-native hot path of fVDB's sparse 3-D networks: index-grid build, kernel map,
sparse convolution forward and backward, transposed convolution, pooling and upsampling (HIP library +
ctypes binding), and what stands around a convolution in a network: norms, gate and residual connection of a block,
dropout, a gated linear recurrence along a grid's voxels, and attention along them with a paged cache for running
sequences."""
from .binding import (FxError, KVCache, Sequences, attention_bwd, attention_fwd, attention_step, cache_read, cache_write, block_join_bwd, block_join_fwd, dropout, gated_scan_bwd, gated_scan_fwd, gated_scan_step, rms_norm_bwd, rms_norm_fwd,  # noqa: F401
                      IndexGrid, KernelMap, build_index_grid, build_index_grid_from_points, build_kernel_map, build_kernel_map_onto, build_sequences, get_option, set_option, use_torch_allocator,  # noqa: F401
                      pool2, pool2_bwd, profile_enable, profile_read, profile_reset, sparse_conv_bwd_data,
                      sparse_conv_bwd_weight, sparse_conv_fwd, sparse_conv_fwd_noalloc, sparse_conv_leaf_bwd_data, sparse_conv_leaf_bwd_weight, sparse_conv_leaf_fwd, sparse_conv_transpose_fwd,
                      upsample2, upsample2_bwd, version)
