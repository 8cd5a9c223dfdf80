"""MI355X-native per-partition data path of VIP-cached, partitioned GNN minibatch preparation.

Four calls, each a thin binding over the C interface in include/spp.h whose work runs in
hand-written HIP kernels for gfx950: vip_propagate, build_vip_cache, sample_mfg,
gather_features.  Beside them what a training loop does with the gathered rows: rows in
4 bits (mx4_quantize), the layer that reads them (mx4_product_multi), its gradient
(mx4_weight_grad) and the optimiser's step (AdamW).
"""
from .api import (access_count, Cache, Context, Graph, LocalStore, MFGBuffers, SppError, build_local_store, build_vip_cache, gather_features, gather_features_multi, gather_features_static, gather_join,  # noqa: F401
                  gather_last_stats, load_library, mfg_bound, release_memory, stream_rates, sample_mfg, sample_mfg_general, sample_mfg_multi, vip_propagate_general, vip_propagate, vip_last_hops, EXPORTS, LIB_PATH,
                  AdamW, RowLists, mx4_dequantize, mx4_product, mx4_product_multi, mx4_quantize, mx4_row_bytes, mx4_weight_grad)
