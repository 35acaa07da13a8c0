"""Batched AES-GCM (AES-256 first of all) for one MI355X: a thin ctypes binding over libpgcm.so.

The binding marshals arguments only; every step of the cipher runs in the library's HIP
kernels.  Importing the package does not load the library; the first call does, and fails
loudly when libpgcm.so has not been built (python -m paper_2411_03357_amd.build).
"""
from .binding import (PgcmError, Key, expand_key, expand_key_bytes, encrypt_batch, decrypt_verify_batch,  # noqa: F401
                      encrypt_batch_keys, decrypt_verify_batch_keys, encrypt_batch_static, reserve,
                      describe_context, describe_schedule, STATIC_WORKSPACE_BYTES, STATIC_MAX_CHUNKS,
                      plan_units, unit_bytes, batch_unit_bytes, library_path, load_library, set_timing, set_unit_bytes, set_one_launch, set_matrix_hash, bitsliced_keystream, copy_key_tables,
                      last_bulk_kernel_ms, bulk_kernel_ms_history, measure_passes, EXPORTS, Sequencer, seq_iv_bytes, SEQ_EXPORTS, BouncePool,
                      BOUNCE_EXPORTS, Pipe, Receiver, PIPE_EXPORTS)

_KV = ("KVCache", "KVWorkspace", "kv_workspace", "kv_append", "kv_attend", "kv_summarize", "kv_select", "kv_evict",
       "KV_EXPORTS")


def __getattr__(name):
    # the operators on KV blocks take torch tensors; what works without torch does not import it
    if name not in _KV:
        raise AttributeError("module %r has no attribute %r" % (__name__, name))
    from . import kv
    globals().update({n: getattr(kv, n) for n in _KV})
    return globals()[name]
