"""The decoder-step structures of include/ilpm.h as packed bytes, for calls of the C ABI from the tests."""
import struct

HEADS = struct.Struct("@Pqqii")                # ilpm_heads
CACHE = struct.Struct("@PPqqqqqqPqiiiiiii4x")  # ilpm_kv_cache
OPTIONS = struct.Struct("@Pqffiii4x")          # ilpm_attn_options
NORM = struct.Struct("@PPPPPPPPPqqqqqiiiiiiiff4x")  # ilpm_residual_norm_args


def heads(t, dtype):
    """A tensor [rows, heads, head_dim]."""
    return HEADS.pack(t.data_ptr(), t.stride(0), t.stride(1), dtype, t.shape[1])


def cache(k, v, table, dtype):
    """Pools [n_pages, page_size, kv_heads, head_dim] and a table [n_seqs, max_pages]."""
    return CACHE.pack(k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3], table.data_ptr(), table.stride(0), dtype,
                      *k.shape, *table.shape)
