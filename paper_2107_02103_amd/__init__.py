"""MI355X (gfx950) implementation of the compressed se_a descriptor of
DP Compress (arXiv:2107.02103): a C-ABI library (libdpc.so, HIP kernels and
a host table builder) and its thin Python binding.

Importing the package does not load the library (so that ``build`` can run
on a fresh tree); the first use of any binding name loads it and raises
ImportError if it has not been built."""
_BINDING = ("DPC_F32", "DPC_F32_ACC64", "DPC_F64", "DPC_OK", "DPC_EINVAL", "DPC_ERANGE",
            "DPC_EHIP", "DPC_ENOTSUP", "DPC_EOVERFLOW", "DPC_NLIST_NOALLOC_MAX_ATOMS", "DpcError", "build_tables", "dpc_build_table",
            "dpc_descriptor_bwd", "dpc_env_mat_a", "dpc_fitting_fwd_bwd", "dpc_fitting_net",
            "dpc_fitting_workspace_bytes", "dpc_force_a", "dpc_last_hip_error", "RocblasHandle",
            "dpc_nlist_reverse", "dpc_nlist_workspace_bytes", "dpc_nlist_build",
            "dpc_nlist_build_noalloc", "dpc_se_a_tab_bwd", "dpc_se_a_tab_bwd_from_dD", "dpc_se_a_tab_fwd", "dpc_strerror",
            "dpc_table_layout", "dpc_version", "make_ranges",
            "DPC_ELEM_F64", "DPC_ELEM_F32", "DPC_ELEM_F16", "DPC_ELEM_BF16", "DPC_MAX_EXPERTS", "DPC_MAX_TOPK",
            "DPC_MAX_I8_COLS", "dpc_route_workspace_bytes", "dpc_route_plan", "dpc_route_gather", "dpc_route_combine",
            "dpc_route_combine_bwd", "dpc_quant_rows", "dpc_matmul_i8", "dpc_linear_i8_workspace_bytes",
            "dpc_linear_i8", "elem_of", "i8_ld",
            "DPC_SCORE_SOFTMAX", "DPC_SCORE_SIGMOID", "DPC_MAX_GATE_GROUPS", "DPC_MAX_MX4_COLS", "dpc_gate_spec", "dpc_gate",
            "dpc_gate_bwd", "dpc_embed", "dpc_embed_bwd_workspace_bytes", "dpc_embed_bwd", "dpc_quant_mx4",
            "dpc_values_mx4", "dpc_matmul_mx4", "dpc_linear_mx4_workspace_bytes", "dpc_linear_mx4", "mx4_ld")
_OBJECTS = {"SeATab": "descriptor", "Route": "experts", "Int8Linear": "experts", "Gate": "gate", "Embedding": "gate",
            "Mx4Rows": "mx4", "Mx4Linear": "mx4"}


def __getattr__(name):
    if name in _BINDING:
        from . import binding
        value = getattr(binding, name)
    elif name in _OBJECTS:
        from importlib import import_module
        value = getattr(import_module("." + _OBJECTS[name], __name__), name)
    else:
        raise AttributeError(name)
    globals()[name] = value              # found without this function from now on (it takes microseconds)
    return value
