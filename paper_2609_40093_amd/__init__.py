"""MI355X-native expert-parallel MoE token dispatch and combine (one rank's share), with the
layer's operators around them.

The work happens in libep.so (HIP kernels for gfx950 plus SDMA host legs; C ABI in
include/ep.h and include/ep_layer.h).  ``paper_2609_40093_amd.api`` is the Python binding of
the first, ``paper_2609_40093_amd.layer`` of the second; the names below are
re-exported lazily so that ``paper_2609_40093_amd.synth`` (input generation only) can be
imported without torch or a GPU.
"""

_API = ("EPError", "Layout", "Staging", "SimPeers", "dispatch_layout", "layout_validate", "dispatch", "dispatch_fused",
        "combine", "trace_enable", "trace_read", "trace_reset", "copy_probe", "stream_probe", "workspace_bytes",
        "pcie_probe",
        "MODE_PER_SENDER", "MODE_DUPLEX", "MODE_REMOTE_ONLY", "MODE_ACCUMULATE", "LocalLayout", "dispatch_layout_local", "pack",
        "combine_rows", "Dense", "allgather", "reducescatter", "round_advance", "round_read", "dispatch_graph",
        "combine_graph", "graph_legs_sdma")

_LAYER = ("Norm", "rmsnorm", "rmsnorm_grad", "rows8_empty", "rows8_values", "Routing", "route", "route_grad",
          "combine_grad", "Product", "expert_product", "ProductGrad", "expert_product_grad")

__all__ = list(_API + _LAYER)


def __getattr__(name):
    if name in _API:
        from . import api
        value = getattr(api, name)
        globals()[name] = value  # later lookups skip this function
        return value
    if name in _LAYER:
        from . import layer
        value = getattr(layer, name)
        globals()[name] = value
        return value
    raise AttributeError(name)
