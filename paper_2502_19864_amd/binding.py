"""ctypes binding of libringada.so (include/ringada.h): same names, argument
marshalling only.  Every function raises RingadaError on a non-OK status,
with the library's message."""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, byref, c_char, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_uint32, c_void_p

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libringada.so")

RINGADA_OK, RINGADA_E_INVALID, RINGADA_E_STATE, RINGADA_E_WORKSPACE, RINGADA_E_UNSUPPORTED, RINGADA_E_HIP = range(6)
ARCH_POSTLN_GELU, ARCH_PRERMS_SWIGLU = 0, 1
F32, BF16 = 0, 1
PLACEMENT_HOULSBY, PLACEMENT_FFN = 0, 1
NORM_LAYER, NORM_RMS = 0, 1
STATUS_NAMES = {0: "OK", 1: "E_INVALID", 2: "E_STATE", 3: "E_WORKSPACE", 4: "E_UNSUPPORTED", 5: "E_HIP"}


class RingadaError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), msg))
        self.status = status


class StageDesc(ctypes.Structure):
    _fields_ = [("arch", c_int32), ("dtype", c_int32), ("n_blocks", c_int32), ("d_model", c_int32),
                ("n_heads", c_int32), ("d_ffn", c_int32), ("d_adapter", c_int32),
                ("max_batch", c_int32), ("max_seq", c_int32), ("norm_eps", c_float),
                ("rope_theta", c_float), ("placement", c_int32)]


class BlockWeights(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("w_qkv", "b_qkv", "w_o", "b_o", "norm1_g", "norm1_b", "w_in",
                                        "b_in", "w_out", "b_out", "norm2_g", "norm2_b")]


class Adapter(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("w_down", "w_up", "g_down", "g_up")]


class Optim(ctypes.Structure):
    _fields_ = [("kind", c_int32), ("lr", c_float)]


class ProfEntry(ctypes.Structure):
    _fields_ = [("name", c_char * 64), ("launches", c_int32), ("total_ms", c_double),
                ("flops", c_double), ("bytes", c_double)]


class View(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("batch", c_int64), ("row", c_int64), ("head", c_int64)]


class AttnDesc(ctypes.Structure):
    _fields_ = [("dtype", c_int32), ("batch", c_int32), ("n_heads", c_int32), ("n_kv_heads", c_int32),
                ("d_head", c_int32), ("seq_q", c_int32), ("seq_k", c_int32), ("causal", c_int32),
                ("window", c_int32), ("sinks", c_int32), ("scale", c_float), ("n_buckets", c_int32),
                ("max_distance", c_int32)]


class AttnTensors(ctypes.Structure):
    _fields_ = [("q", View), ("k", View), ("v", View), ("o", View), ("lse", c_void_p), ("len_q", c_void_p),
                ("len_k", c_void_p), ("table", c_void_p), ("bucket", c_void_p)]


class StageAttention(ctypes.Structure):
    _fields_ = [("window", c_int32), ("sinks", c_int32), ("n_buckets", c_int32), ("max_distance", c_int32),
                ("table", c_void_p), ("bucket", c_void_p), ("g_table", c_void_p), ("workspace", c_void_p),
                ("workspace_bytes", c_size_t)]


class AttnGrads(ctypes.Structure):
    _fields_ = [("dout", View), ("dq", View), ("dk", View), ("dv", View), ("dtable", c_void_p)]


class Rows(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("row", c_int64)]


class NormDesc(ctypes.Structure):
    _fields_ = [("dtype", c_int32), ("kind", c_int32), ("rows", c_int64), ("d", c_int32), ("eps", c_float)]


class RotaryDesc(ctypes.Structure):
    _fields_ = [("dtype", c_int32), ("batch", c_int32), ("rows", c_int32), ("n_heads", c_int32),
                ("n_kv_heads", c_int32), ("d_head", c_int32), ("n_axes", c_int32), ("section", c_int32 * 4),
                ("inverse", c_int32)]


class VocabDesc(ctypes.Structure):
    _fields_ = [("dtype", c_int32), ("rows", c_int32), ("d", c_int32), ("vocab", c_int32)]


class VocabTensors(ctypes.Structure):
    _fields_ = [("h", Rows), ("w", Rows), ("labels", c_void_p), ("loss", c_void_p), ("lse", c_void_p),
                ("dloss", c_void_p), ("dh", Rows), ("dw", Rows)]


# (name, restype, argtypes): every symbol declared in include/ringada.h
SIGNATURES = [
    ("ringada_stage_plan", c_int32, [POINTER(StageDesc), c_int32, c_int32, c_int32,
                                     POINTER(c_size_t), POINTER(c_size_t)]),
    ("ringada_local_cutoff", c_int32, [c_int32, c_int32, c_int32, c_int32]),
    ("ringada_stage_plan_weights", c_int32, [POINTER(StageDesc), POINTER(c_size_t), POINTER(c_size_t)]),
    ("ringada_stage_create", c_int32, [POINTER(StageDesc), c_void_p, c_size_t, POINTER(c_void_p)]),
    ("ringada_stage_bind_block", c_int32, [c_void_p, c_int32, POINTER(BlockWeights), POINTER(Adapter),
                                           POINTER(Adapter), c_void_p, c_size_t, c_void_p]),
    ("ringada_stage_sync_adapters", c_int32, [c_void_p, c_void_p]),
    ("ringada_stage_destroy", None, [c_void_p]),
    ("ringada_stage_plan_attention", c_int32, [POINTER(StageDesc), POINTER(StageAttention), c_int32, c_int32,
                                               POINTER(c_size_t)]),
    ("ringada_stage_set_attention", c_int32, [c_void_p, POINTER(StageAttention)]),
    ("ringada_stage_set_dropout", c_int32, [c_void_p, c_float, c_void_p, c_uint32]),
    ("ringada_stage_forward", c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32,
                                        c_void_p, c_size_t, c_void_p, c_size_t]),
    ("ringada_stage_backward", c_int32, [c_void_p, c_void_p, c_void_p, c_int32, c_void_p]),
    ("ringada_adapter_step", c_int32, [c_void_p, c_void_p, c_int32, POINTER(Optim)]),
    ("ringada_loss_mse", c_int32, [c_void_p, c_int32, c_void_p, c_void_p, c_int64, c_void_p, c_void_p]),
    ("ringada_head_ce", c_int32, [c_void_p, c_int32, c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p,
                                  c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    ("ringada_sgd_f32", c_int32, [c_void_p, c_void_p, c_void_p, c_int64, c_float]),
    ("ringada_attn_plan", c_int32, [c_void_p, c_int32, POINTER(c_size_t), POINTER(c_size_t)]),
    # the structs may come as the ctypes structures or packed into bytes
    ("ringada_attn_forward", c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_size_t]),
    ("ringada_attn_backward", c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t]),
    ("ringada_relpos_buckets", c_int32, [c_int32, c_int32, c_int32, POINTER(c_int32)]),
    ("ringada_dropout", c_int32, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_int64, c_float, c_void_p,
                                  c_uint32]),
    ("ringada_norm_forward", c_int32, [c_void_p] * 9),
    ("ringada_norm_plan", c_int32, [c_void_p, POINTER(c_size_t)]),
    ("ringada_norm_backward", c_int32, [c_void_p] * 11 + [c_size_t]),
    ("ringada_rotary", c_int32, [c_void_p] * 8),
    ("ringada_rotary_frequencies", c_int32, [c_int32, POINTER(c_int32), c_double, c_int32, POINTER(c_double)]),
    ("ringada_vocab_plan", c_int32, [c_void_p, POINTER(c_size_t), POINTER(c_size_t), POINTER(c_size_t)]),
    ("ringada_vocab_ce", c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_size_t]),
    ("ringada_vocab_next", c_int32, [c_void_p] * 7 + [c_size_t]),
    ("ringada_last_error", c_char_p, []),
    ("ringada_prof_begin", c_int32, [c_void_p]),
    ("ringada_prof_end", c_int32, [c_void_p, POINTER(ProfEntry), c_int32, POINTER(c_int32)]),
]

_lib = None


def lib():
    """Loads libringada.so (built in-tree); raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libringada.so is not built (run `python -m paper_2502_19864_amd.build`); "
                               "there is no fallback implementation")
        L = ctypes.CDLL(LIB_PATH)
        for name, res, args in SIGNATURES:
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(status):
    if status != RINGADA_OK:
        msg = lib().ringada_last_error()
        raise RingadaError(status, msg.decode() if msg else "")


def _p(x):
    """Device pointer of a torch tensor, an int address or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _ref(x):
    """A structure by reference, or its packed bytes (or None) as they are."""
    return x if type(x) is bytes or x is None else byref(x)


def _in(name, x, low, bits):
    """x, an integer from low to 2^bits - 1: ctypes would cut others to their low bits."""
    if not low <= x < 1 << bits:
        raise ValueError(f"{name}: {x} is out of range")
    return x


def ringada_stage_plan(desc, batch, seq, lowest_unfrozen):
    st, sc = c_size_t(0), c_size_t(0)
    _check(lib().ringada_stage_plan(byref(desc), batch, seq, lowest_unfrozen, byref(st), byref(sc)))
    return st.value, sc.value


def ringada_local_cutoff(n_tm, depth, first_block, n_local):
    return lib().ringada_local_cutoff(n_tm, depth, first_block, n_local)


def ringada_stage_plan_weights(desc):
    blk, stg = c_size_t(0), c_size_t(0)
    _check(lib().ringada_stage_plan_weights(byref(desc), byref(blk), byref(stg)))
    return blk.value, stg.value


def ringada_stage_create(desc, stage_mem, stage_mem_bytes):
    h = c_void_p()
    _check(lib().ringada_stage_create(byref(desc), _p(stage_mem), stage_mem_bytes, byref(h)))
    return h


def ringada_stage_bind_block(stage, block, frozen, attn_adapter, ffn_adapter, block_mem, block_mem_bytes, stream):
    """attn_adapter is None for a stage with the single (FFN) placement."""
    _check(lib().ringada_stage_bind_block(stage, block, byref(frozen),
                                          None if attn_adapter is None else byref(attn_adapter),
                                          byref(ffn_adapter), _p(block_mem), block_mem_bytes, stream))


def ringada_stage_sync_adapters(stage, stream):
    _check(lib().ringada_stage_sync_adapters(stage, stream))


def ringada_stage_destroy(stage):
    lib().ringada_stage_destroy(stage)


def ringada_stage_plan_attention(desc, opt, batch, seq):
    n = c_size_t(0)
    _check(lib().ringada_stage_plan_attention(byref(desc), byref(opt), batch, seq, byref(n)))
    return n.value


def ringada_stage_set_attention(stage, opt):
    """opt None: the plain attention."""
    _check(lib().ringada_stage_set_attention(stage, None if opt is None else byref(opt)))


def ringada_stage_set_dropout(stage, p, rng, first_site):
    _check(lib().ringada_stage_set_dropout(stage, p, _p(rng), _in("first_site", first_site, 0, 32)))


def ringada_stage_forward(stage, stream, x, y, batch, seq, lowest_unfrozen, stash, stash_bytes, scratch,
                          scratch_bytes):
    _check(lib().ringada_stage_forward(stage, stream, _p(x), _p(y), batch, seq, lowest_unfrozen, _p(stash),
                                       stash_bytes, _p(scratch), scratch_bytes))


def ringada_stage_backward(stage, stream, dy, lowest_unfrozen, dx_in):
    _check(lib().ringada_stage_backward(stage, stream, _p(dy), lowest_unfrozen, _p(dx_in)))


def ringada_adapter_step(stage, stream, lowest_unfrozen, lr, kind=0):
    opt = Optim(kind, lr)
    _check(lib().ringada_adapter_step(stage, stream, lowest_unfrozen, byref(opt)))


def ringada_loss_mse(stream, dtype, y, target, n, dy, loss):
    _check(lib().ringada_loss_mse(stream, dtype, _p(y), _p(target), n, _p(dy), _p(loss)))


def ringada_head_ce(stream, dtype, y, batch, seq, d, w_h, b_h, n_classes, labels, dy, g_wh, g_bh, loss):
    _check(lib().ringada_head_ce(stream, dtype, _p(y), batch, seq, d, _p(w_h), _p(b_h), n_classes, _p(labels),
                                 _p(dy), _p(g_wh), _p(g_bh), _p(loss)))


def ringada_sgd_f32(stream, w, g, n, lr):
    _check(lib().ringada_sgd_f32(stream, _p(w), _p(g), n, lr))


def ringada_attn_plan(desc, with_dtable):
    f, b = c_size_t(0), c_size_t(0)
    _check(lib().ringada_attn_plan(_ref(desc), int(with_dtable), byref(f), byref(b)))
    return f.value, b.value


def ringada_attn_forward(stream, desc, tensors, workspace, workspace_bytes):
    _check(lib().ringada_attn_forward(stream, _ref(desc), _ref(tensors), _p(workspace), workspace_bytes))


def ringada_attn_backward(stream, desc, tensors, grads, workspace, workspace_bytes):
    _check(lib().ringada_attn_backward(stream, _ref(desc), _ref(tensors), _ref(grads), _p(workspace), workspace_bytes))


def ringada_relpos_buckets(n_buckets, max_distance, bidirectional):
    """The map as a list of 2 max_distance + 1 ints, indexed by key - query + max_distance."""
    _in("n_buckets", n_buckets, -1 << 31, 31)
    _in("max_distance", max_distance, -1 << 31, 16)  # the library takes 1024
    m = (c_int32 * max(1, 2 * max_distance + 1))()
    _check(lib().ringada_relpos_buckets(n_buckets, max_distance, int(bidirectional), m))
    return list(m)


def ringada_dropout(stream, dtype, x, res, y, n, p, rng, site):
    _check(lib().ringada_dropout(stream, dtype, _p(x), _p(res), _p(y), _in("n", n, -1 << 63, 63), p, _p(rng),
                                 _in("site", site, 0, 32)))


def ringada_norm_forward(stream, desc, x, res, sum_, gain, shift, y, stats):
    _check(lib().ringada_norm_forward(stream, _ref(desc), _ref(x), _ref(res), _ref(sum_), _p(gain), _p(shift), _ref(y),
                                      _p(stats)))


def ringada_norm_plan(desc):
    n = c_size_t(0)
    _check(lib().ringada_norm_plan(_ref(desc), byref(n)))
    return n.value


def ringada_norm_backward(stream, desc, dy, dskip, sum_, gain, stats, dx, dgain, dshift, workspace, workspace_bytes):
    _check(lib().ringada_norm_backward(stream, _ref(desc), _ref(dy), _ref(dskip), _ref(sum_), _p(gain), _p(stats),
                                       _ref(dx), _p(dgain), _p(dshift), _p(workspace), workspace_bytes))


def ringada_rotary(stream, desc, q, k, positions, freq, q_out, k_out):
    _check(lib().ringada_rotary(stream, _ref(desc), _ref(q), _ref(k), _p(positions), _p(freq), _ref(q_out),
                                _ref(k_out)))


def ringada_rotary_frequencies(sections, theta, shared):
    """The frequencies as a list of sum(sections) floats."""
    if not 1 <= len(sections) <= 4:
        raise ValueError("sections: one to four axes")
    for m in sections:
        _in("section", m, 1, 10)
    s = (c_int32 * len(sections))(*sections)
    f = (c_double * sum(sections))()
    _check(lib().ringada_rotary_frequencies(len(sections), s, theta, int(shared), f))
    return list(f)


def ringada_vocab_plan(desc):
    """Workspace bytes of a call without gradients, of one with, and of ringada_vocab_next."""
    f, t, n = c_size_t(0), c_size_t(0), c_size_t(0)
    _check(lib().ringada_vocab_plan(_ref(desc), byref(f), byref(t), byref(n)))
    return f.value, t.value, n.value


def ringada_vocab_ce(stream, desc, tensors, workspace, workspace_bytes):
    _check(lib().ringada_vocab_ce(stream, _ref(desc), _ref(tensors), _p(workspace), workspace_bytes))


def ringada_vocab_next(stream, desc, h, w, token, logprob, workspace, workspace_bytes):
    _check(lib().ringada_vocab_next(stream, _ref(desc), _ref(h), _ref(w), _p(token), _p(logprob), _p(workspace),
                                    workspace_bytes))


def ringada_last_error():
    m = lib().ringada_last_error()
    return m.decode() if m else ""


def ringada_prof_begin(stage):
    _check(lib().ringada_prof_begin(stage))


def ringada_prof_end(stage, max_entries=64):
    arr = (ProfEntry * max_entries)()
    n = c_int32(0)
    _check(lib().ringada_prof_end(stage, arr, max_entries, byref(n)))
    return [dict(name=arr[i].name.decode(), launches=arr[i].launches, total_ms=arr[i].total_ms,
                 flops=arr[i].flops, bytes=arr[i].bytes) for i in range(min(n.value, max_entries))]
