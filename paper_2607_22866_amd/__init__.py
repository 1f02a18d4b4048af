"""MI355X (gfx950) SpGEMM C = A*B on CSR with the gMAGNUS heavy-row method, and
the products that a sparse routing matrix selects (layers of experts).

The compute lives in libgmagnus.so (HIP kernels behind the C ABI declared in
include/gmagnus.h); :mod:`paper_2607_22866_amd.gmagnus` is its ctypes binding.
"""
from .gmagnus import (DeviceCSR, GmagnusError, Plan, Routing, combine, combine_backward, get_params, group_outer,
                      group_product, group_product_fp8, load, quantise_blocks, release_cache, route, route_backward,
                      row_products, spgemm, split_panels)

__all__ = ["DeviceCSR", "GmagnusError", "Plan", "Routing", "combine", "combine_backward", "get_params", "group_outer",
           "group_product", "group_product_fp8", "load", "quantise_blocks", "release_cache", "route", "route_backward",
           "row_products", "spgemm", "split_panels"]
