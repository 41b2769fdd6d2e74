"""ctypes binding of libtokencarve.so: same names as the C ABI, argument marshalling only.

Every function takes torch tensors that already live on the GPU (contiguous, the
dtype the C header states), passes their device pointers through, and returns
nothing; a non-zero tc_status raises TokenCarveError.  Work is enqueued on
torch's current stream unless `stream` (a raw hipStream_t integer) is given.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtokencarve.so")

TC_F32, TC_BF16, TC_F16 = 0, 1, 2
_DTYPES = {"f32": TC_F32, "bf16": TC_BF16, "f16": TC_F16}
TC_NORM_NONE, TC_NORM_MINMAX = 0, 1
TC_EIG_F64, TC_EIG_F32 = 0, 1
TC_EIG_AUTO, TC_EIG_JACOBI, TC_EIG_TRIDIAGONAL = 0, 1, 2
TC_ROPE_HALF, TC_ROPE_INTERLEAVED = 0, 1
TC_ROPE_PLAIN, TC_ROPE_LINEAR, TC_ROPE_BASE, TC_ROPE_BANDS = 0, 1, 2, 3

SYMBOLS = ("tc_workspace_bytes", "tc_status_string", "tc_attn_output", "tc_ipgs_score", "tc_select_topk",
           "tc_merge", "tc_merge_noalloc", "tc_similarity", "tc_compress", "tc_profile_compress", "tc_probe_rates", "tc_info_rank",
           "tc_assemble_sequence", "tc_kv_cache_fraction", "tc_rope_tables", "tc_rope_apply",
           "tc_cache_workspace_bytes", "tc_cache_append", "tc_cache_attention", "tc_cache_evict")
PROF_KINDS = ("attn", "attn_reduce", "gram", "jacobi_init", "jacobi_solve", "jacobi_update", "jacobi_update_u", "jacobi_sweep_end",
              "sigma", "ics", "combine", "topk", "rownorm", "sim", "assign", "average", "tridiag", "bisect", "twisted",
              "backtransform", "tridiag_update")


class TokenCarveError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("libtokencarve: %s (status %d)" % (text, status))
        self.status = status


class tc_params(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("seq_len", ctypes.c_int32), ("vis_start", ctypes.c_int32),
        ("n_vis", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("hidden_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float), ("lambda_", ctypes.c_float), ("norm_mode", ctypes.c_int32),
        ("sv_rtol", ctypes.c_float), ("k_prune", ctypes.c_int32), ("k_final", ctypes.c_int32),
        ("jacobi_max_sweeps", ctypes.c_int32), ("jacobi_tol", ctypes.c_float), ("eig_dtype", ctypes.c_int32),
        ("eig_method", ctypes.c_int32), ("stream_groups", ctypes.c_int32), ("n_prompt_queries", ctypes.c_int32),
    ]


def make_params(batch, seq_len, vis_start, n_vis, n_heads, head_dim, hidden_dim, dtype, k_prune, k_final,
                lam=0.5, causal=1, norm_mode=TC_NORM_MINMAX, sv_rtol=0.0, softmax_scale=0.0,
                jacobi_max_sweeps=0, jacobi_tol=0.0, eig_dtype=TC_EIG_F64, stream_groups=0, eig_method=0,
                n_prompt_queries=0):
    return tc_params(batch, seq_len, vis_start, n_vis, n_heads, head_dim, hidden_dim, dtype, causal,
                     softmax_scale, lam, norm_mode, sv_rtol, k_prune, k_final, jacobi_max_sweeps, jacobi_tol,
                     eig_dtype, eig_method, stream_groups, n_prompt_queries)


def params_for(w, batch=None, **overrides):
    """tc_params for a workloads.Workload."""
    kw = dict(batch=w.batch if batch is None else batch, seq_len=w.seq_len, vis_start=w.n_sys, n_vis=w.n_vis,
              n_heads=w.n_heads, head_dim=w.head_dim, hidden_dim=w.hidden,
              dtype=_DTYPES[w.dtype], k_prune=w.k_prune, k_final=w.k_final, lam=w.lam,
              causal=w.causal)
    kw.update(overrides)
    return make_params(**kw)


class tc_rope(ctypes.Structure):
    _fields_ = [
        ("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("scaling", ctypes.c_int32),
        ("base", ctypes.c_float), ("factor", ctypes.c_float), ("original_len", ctypes.c_int32), ("low", ctypes.c_float),
        ("high", ctypes.c_float), ("magnitude", ctypes.c_float),
    ]


class tc_strides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("head", ctypes.c_int64), ("row", ctypes.c_int64)]


class tc_cache(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("n_query", ctypes.c_int32), ("capacity", ctypes.c_int32), ("max_len", ctypes.c_int32),
        ("n_prefixes", ctypes.c_int32), ("prefix_len", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
        ("budget", ctypes.c_int32), ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32),
    ]


def make_cache(batch, n_heads, n_kv_heads, head_dim, dtype, n_query, capacity, max_len=0, n_prefixes=0, prefix_len=0,
               softmax_scale=0.0, budget=0, n_sink=0, n_recent=0):
    return tc_cache(batch, n_heads, n_kv_heads, head_dim, dtype, n_query, capacity, max_len, n_prefixes, prefix_len, softmax_scale,
                    budget, n_sink, n_recent)


def make_rope(head_dim, rot_dim=0, layout=TC_ROPE_HALF, scaling=TC_ROPE_PLAIN, base=10000.0, factor=1.0, original_len=0, low=0.0,
              high=0.0, magnitude=0.0):
    return tc_rope(head_dim, rot_dim, layout, scaling, base, factor, original_len, low, high, magnitude)


_lib = None


def load_library():
    """Load libtokencarve.so (built by `python -m paper_2503_10501_amd.build`); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("%s not found: build it with `python -m paper_2503_10501_amd.build` "
                          "(there is no CPU fallback)" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, pp = ctypes.c_void_p, ctypes.c_size_t, ctypes.POINTER(tc_params)
    lib.tc_workspace_bytes.restype = sz
    lib.tc_workspace_bytes.argtypes = [pp]
    lib.tc_status_string.restype = ctypes.c_char_p
    lib.tc_status_string.argtypes = [ctypes.c_int]
    lib.tc_attn_output.argtypes = [pp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tc_ipgs_score.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tc_select_topk.argtypes = [pp, vp, vp, vp, sz, vp]
    lib.tc_merge.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tc_merge_noalloc.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp]
    lib.tc_similarity.argtypes = [pp, vp, vp, vp, vp, sz, vp]
    lib.tc_compress.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tc_profile_compress.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp, vp, vp, ctypes.c_int32, vp]
    lib.tc_probe_rates.argtypes = [vp, sz, vp, vp]
    lib.tc_info_rank.argtypes = [pp, vp, vp, ctypes.c_int32, ctypes.c_float, vp, vp, vp, vp, sz, vp]
    lib.tc_assemble_sequence.argtypes = [pp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp]
    lib.tc_kv_cache_fraction.argtypes = [ctypes.c_int32] * 5
    rp, sp, i32 = ctypes.POINTER(tc_rope), ctypes.POINTER(tc_strides), ctypes.c_int32
    lib.tc_rope_tables.argtypes = [rp, vp, ctypes.c_int64, vp, vp, vp]
    lib.tc_rope_apply.argtypes = [rp, i32, i32, i32, i32, vp, sp, vp, vp, vp, sp, i32, vp]
    cp = ctypes.POINTER(tc_cache)
    lib.tc_cache_workspace_bytes.argtypes = [cp]
    lib.tc_cache_append.argtypes = [cp, rp, vp, sp, vp, sp, vp, sp] + [vp] * 11
    lib.tc_cache_attention.argtypes = [cp] + [vp] * 10 + [sz, vp]
    lib.tc_cache_evict.argtypes = [cp] + [vp] * 9 + [i32, vp, vp, sz, vp]
    for name in SYMBOLS[2:]:
        getattr(lib, name).restype = ctypes.c_int
    lib.tc_cache_workspace_bytes.restype = sz
    lib.tc_kv_cache_fraction.restype = ctypes.c_double
    _lib = lib
    return lib


def _ptr(t, dtype=None):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous and on the GPU")
    if dtype is not None and t.dtype != dtype:
        raise ValueError("expected %s, got %s" % (dtype, t.dtype))
    return t.data_ptr()


def _stream(stream):
    return torch.cuda.current_stream().cuda_stream if stream is None else stream


def _check(rc):
    if rc != 0:
        raise TokenCarveError(rc, load_library().tc_status_string(rc).decode())


def storage_dtype(p):
    return {TC_F32: torch.float32, TC_BF16: torch.bfloat16, TC_F16: torch.float16}[p.dtype]


def tc_status_string(status):
    return load_library().tc_status_string(status).decode()


def tc_workspace_bytes(p):
    return int(load_library().tc_workspace_bytes(ctypes.byref(p)))


def new_workspace(p, device="cuda"):
    n = tc_workspace_bytes(p)
    if n == 0:
        raise TokenCarveError(-4, "invalid tc_params")
    return torch.empty(n, dtype=torch.uint8, device=device)


def tc_attn_output(p, Q, K, V, O, attn_score, ws, stream=None):
    sd = storage_dtype(p)
    _check(load_library().tc_attn_output(ctypes.byref(p), _ptr(Q, sd), _ptr(K, sd), _ptr(V, sd), _ptr(O, sd),
                                         _ptr(attn_score, torch.float32), _ptr(ws), ws.numel(), _stream(stream)))


def tc_ipgs_score(p, O, attn_score, score, ics, sigma, info, ws, stream=None):
    sd = storage_dtype(p)
    _check(load_library().tc_ipgs_score(ctypes.byref(p), _ptr(O, sd), _ptr(attn_score, torch.float32),
                                        _ptr(score, torch.float32), _ptr(ics, torch.float32),
                                        _ptr(sigma, torch.float32), _ptr(info, torch.int32), _ptr(ws), ws.numel(),
                                        _stream(stream)))


def tc_select_topk(p, score, order, ws, stream=None):
    _check(load_library().tc_select_topk(ctypes.byref(p), _ptr(score, torch.float32), _ptr(order, torch.int32),
                                         _ptr(ws), ws.numel(), _stream(stream)))


def tc_merge(p, X, metric, order, X_out, kept_idx, merge_dst, ws, stream=None):
    sd = storage_dtype(p)
    _check(load_library().tc_merge(ctypes.byref(p), _ptr(X, sd), _ptr(metric, sd), _ptr(order, torch.int32),
                                   _ptr(X_out, sd), _ptr(kept_idx, torch.int32), _ptr(merge_dst, torch.int32),
                                   _ptr(ws), ws.numel(), _stream(stream)))


def tc_merge_noalloc(p, X, metric, order, X_out, kept_idx, merge_dst, stream=None):
    sd = storage_dtype(p)
    _check(load_library().tc_merge_noalloc(ctypes.byref(p), _ptr(X, sd), _ptr(metric, sd), _ptr(order, torch.int32),
                                           _ptr(X_out, sd), _ptr(kept_idx, torch.int32),
                                           _ptr(merge_dst, torch.int32), _stream(stream)))


def tc_similarity(p, metric, order, sim, ws, stream=None):
    _check(load_library().tc_similarity(ctypes.byref(p), _ptr(metric, storage_dtype(p)), _ptr(order, torch.int32),
                                        _ptr(sim, torch.float32), _ptr(ws), ws.numel(), _stream(stream)))


def tc_compress(p, Q, K, V, X, X_out, kept_idx, merge_dst, ws, O=None, score=None, order=None, info=None,
                stream=None):
    sd = storage_dtype(p)
    _check(load_library().tc_compress(ctypes.byref(p), _ptr(Q, sd), _ptr(K, sd), _ptr(V, sd), _ptr(X, sd),
                                      _ptr(X_out, sd), _ptr(kept_idx, torch.int32), _ptr(merge_dst, torch.int32),
                                      _ptr(O, sd), _ptr(score, torch.float32), _ptr(order, torch.int32),
                                      _ptr(info, torch.int32), _ptr(ws), ws.numel(), _stream(stream)))


def tc_profile_compress(p, Q, K, V, X, X_out, kept_idx, merge_dst, info, ws, max_sweeps_out=64, stream=None):
    """Returns ({kind: (total_ms, launches)}, [jacobi_update ms per sweep]); blocks until the stream is idle.
    The extra keys "jacobi_update_tiles" and "jacobi_rotation_steps" hold (0.0, count): the 64x64 tiles the
    tile update processed and the rotation steps the rotation kernel applied."""
    sd = storage_dtype(p)
    n = len(PROF_KINDS)
    ms = (ctypes.c_float * n)()
    cnt = (ctypes.c_int32 * n)()
    per_sweep = (ctypes.c_float * max_sweeps_out)()
    work = (ctypes.c_int64 * 2)()
    _check(load_library().tc_profile_compress(ctypes.byref(p), _ptr(Q, sd), _ptr(K, sd), _ptr(V, sd), _ptr(X, sd),
                                              _ptr(X_out, sd), _ptr(kept_idx, torch.int32),
                                              _ptr(merge_dst, torch.int32), _ptr(info, torch.int32), _ptr(ws),
                                              ws.numel(), _stream(stream), ms, cnt, per_sweep, max_sweeps_out,
                                              work))
    kinds = {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(PROF_KINDS)}
    kinds["jacobi_update_tiles"] = (0.0, int(work[0]))
    kinds["jacobi_rotation_steps"] = (0.0, int(work[1]))
    return kinds, [float(x) for x in per_sweep]


def tc_probe_rates(stream=None):
    """Sustained {fp64, fp32, bf16} matrix-core TFLOP/s and streaming-copy GB/s of the current GPU."""
    ws = torch.empty(1 << 31, dtype=torch.uint8, device="cuda")
    rates = (ctypes.c_float * 5)()
    _check(load_library().tc_probe_rates(_ptr(ws), ws.numel(), _stream(stream), rates))
    return {"mfma_f64_tflops": float(rates[0]), "mfma_f32_tflops": float(rates[1]),
            "mfma_bf16_tflops": float(rates[2]), "copy_gbps": float(rates[3]),
            "mfma_f64_4x4x4_tflops": float(rates[4])}


def tc_info_rank(p, O, rank, ws, rows=None, rtol=0.0, sigma=None, info=None, stream=None):
    n_rows = int(rows.shape[1]) if rows is not None else int(p.n_vis)
    if rows is not None and rows.numel() == 0:   # an empty tensor has no address; NULL would mean "all rows"
        rows = torch.zeros(4, dtype=torch.int32, device="cuda")
    _check(load_library().tc_info_rank(ctypes.byref(p), _ptr(O), _ptr(rows, torch.int32), n_rows, float(rtol),
                                       _ptr(rank, torch.int32), _ptr(sigma, torch.float32), _ptr(info, torch.int32),
                                       _ptr(ws), ws.numel(), _stream(stream)))


def tc_assemble_sequence(p, H, X_out, kept_idx, H_new, pos_ids, rope_base=10000.0, rope_cos=None, rope_sin=None,
                         stream=None):
    _check(load_library().tc_assemble_sequence(ctypes.byref(p), _ptr(H), _ptr(X_out), _ptr(kept_idx, torch.int32),
                                               _ptr(H_new), _ptr(pos_ids, torch.int32), float(rope_base),
                                               _ptr(rope_cos, torch.float32), _ptr(rope_sin, torch.float32),
                                               _stream(stream)))


def tc_kv_cache_fraction(n_text, n_vis, n_kept, n_layers, n_layers_before):
    return float(load_library().tc_kv_cache_fraction(n_text, n_vis, n_kept, n_layers, n_layers_before))


# ---- behind the compression: the tensors' shapes are checked, and work goes to the device that holds them.  A decoding step makes these
# calls for every layer: they keep to what a check costs (14 tensors: 5 us).

_I32, _F32, _U8 = torch.int32, torch.float32, torch.uint8
_STORAGE = {TC_F32: torch.float32, TC_BF16: torch.bfloat16, TC_F16: torch.float16}
_CODES = {v: k for k, v in _STORAGE.items()}


def _refuse(name, t, shape, dtype, dev):
    if t.dtype != dtype:
        raise ValueError("%s: expected %s, got %s" % (name, dtype, t.dtype))
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s: expected shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if t.get_device() != dev or dev < 0:
        raise ValueError("%s: tensors must be on one GPU" % name)
    raise ValueError("%s: must be contiguous" % name)


def _whole(name, t, shape, dtype, dev):
    """Address of a contiguous tensor (None for None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _refuse(name, t, shape, dtype, dev)
    return t.data_ptr()


def _rows(name, t, shape, dtype, dev):
    """Address and strides of a [batch, head, row, d_h] view with contiguous rows."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        _refuse(name, t, shape, dtype, dev)
    b, h, r, e = t.stride()
    if e != 1:
        raise ValueError("%s: the elements of a row must be contiguous" % name)
    return t.data_ptr(), ctypes.byref(tc_strides(b, h, r))


def _device(name, t):
    dev = t.get_device()
    if dev < 0:
        raise ValueError("%s: tensors must be on the GPU" % name)
    return dev


def _call(entry, dev, stream, *args):
    """The entry point on the device that holds the tensors: on its current stream, or the caller's."""
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(dev)
    if dev == torch._C._cuda_getDevice():
        rc = entry(*args, stream)
    else:
        with torch.cuda.device(dev):
            rc = entry(*args, stream)
    if rc != 0:
        _check(rc)


def _rot(r):
    return r.rot_dim if r.rot_dim > 0 else r.head_dim


def tc_rope_tables(r, pos_ids, cos, sin, stream=None):
    """cos, sin: the shape of pos_ids and r/2 behind it."""
    dev, shape = _device("pos_ids", pos_ids), pos_ids.shape
    tables = (*shape, _rot(r) // 2)
    _call(load_library().tc_rope_tables, dev, stream, r, _whole("pos_ids", pos_ids, shape, _I32, dev), pos_ids.numel(),
          _whole("cos", cos, tables, _F32, dev), _whole("sin", sin, tables, _F32, dev))


def tc_rope_apply(r, x, cos, sin, y=None, transposed=False, stream=None):
    """x, y: [batch, heads, rows, head_dim] views; without y the rows of x are turned in place.  No call of this module is recorded for
    gradients; this one, whose gradient is the transposed turn, refuses tensors that require them unless they are switched off (torch.no_grad)."""
    if torch.is_grad_enabled() and (x.requires_grad or (y is not None and y.requires_grad)):
        raise ValueError("x, y: the turn is not recorded for gradients: call it under torch.no_grad(), its gradient is transposed=True")
    dev, sd, shape = _device("x", x), x.dtype, x.shape
    if x.dim() != 4 or shape[3] != r.head_dim:
        raise ValueError("x: expected [batch, heads, rows, %d], got %s" % (r.head_dim, tuple(shape)))
    if sd not in _CODES:
        raise ValueError("x: %s is no storage type" % sd)
    B, H, T, _ = shape
    px, xs = _rows("x", x, shape, sd, dev)
    py, ys = (px, xs) if y is None else _rows("y", y, shape, sd, dev)
    tables = (B, T, _rot(r) // 2)
    _call(load_library().tc_rope_apply, dev, stream, r, _CODES[sd], B, H, T, px, xs, _whole("cos", cos, tables, _F32, dev),
          _whole("sin", sin, tables, _F32, dev), py, ys, int(transposed))


def tc_cache_workspace_bytes(c):
    return int(load_library().tc_cache_workspace_bytes(ctypes.byref(c)))


def new_cache_workspace(c, device="cuda"):
    n = tc_cache_workspace_bytes(c)
    if n == 0:
        raise TokenCarveError(-4, "invalid tc_cache")
    return torch.empty(n, dtype=torch.uint8, device=device)


def tc_cache_append(c, r, Q, K, V, cos, sin, pos_ids, lens, Q_out, K_cache, V_cache, slot_pos, weight, q_len=None, stream=None):
    """Q [B, H, T, d], K, V [B, H_kv, T, d]: views; r, cos and sin None: nothing is turned."""
    dev, sd = _device("Q", Q), _STORAGE[c.dtype]
    B, H, Hk, T, d, cap = c.batch, c.n_heads, c.n_kv_heads, c.n_query, c.head_dim, c.capacity
    tables, slots, rows = (B, T, _rot(r) // 2 if r is not None else 0), (B, Hk, cap), (B, Hk, T, d)
    q, qs = _rows("Q", Q, (B, H, T, d), sd, dev)
    k, ks = _rows("K", K, rows, sd, dev)
    v, vs = _rows("V", V, rows, sd, dev)
    cache = (B, Hk, cap, d)
    _call(load_library().tc_cache_append, dev, stream, c, r, q, qs, k, ks, v, vs, _whole("cos", cos, tables, _F32, dev),
          _whole("sin", sin, tables, _F32, dev), _whole("pos_ids", pos_ids, (B, T), _I32, dev), _whole("lens", lens, (B,), _I32, dev),
          _whole("q_len", q_len, (B,), _I32, dev), _whole("Q_out", Q_out, (B, H, T, d), sd, dev), _whole("K_cache", K_cache, cache, sd, dev),
          _whole("V_cache", V_cache, cache, sd, dev), _whole("slot_pos", slot_pos, slots, _I32, dev),
          _whole("weight", weight, slots, _F32, dev))


def tc_cache_attention(c, Q, K_cache, V_cache, lens, O, ws, K_prefix=None, V_prefix=None, weight=None, q_len=None, stream=None):
    dev, sd = _device("Q", Q), _STORAGE[c.dtype]
    B, H, Hk, T, d, cap = c.batch, c.n_heads, c.n_kv_heads, c.n_query, c.head_dim, c.capacity
    cache, prefix = (B, Hk, cap, d), (c.n_prefixes, Hk, c.prefix_len, d)
    if prefix[2] > 0 and (K_prefix is None or V_prefix is None):
        raise ValueError("K_prefix, V_prefix: expected shape %s" % (prefix,))
    _call(load_library().tc_cache_attention, dev, stream, c, _whole("Q", Q, (B, H, T, d), sd, dev),
          _whole("K_prefix", K_prefix, prefix, sd, dev), _whole("V_prefix", V_prefix, prefix, sd, dev),
          _whole("K_cache", K_cache, cache, sd, dev), _whole("V_cache", V_cache, cache, sd, dev), _whole("lens", lens, (B,), _I32, dev),
          _whole("q_len", q_len, (B,), _I32, dev), _whole("O", O, (B, T, H * d), sd, dev), _whole("weight", weight, (B, Hk, cap), _F32, dev),
          _whole("ws", ws, (ws.numel(),), _U8, dev), ws.numel())


def tc_cache_evict(c, lens, K_cache, V_cache, slot_pos, weight, len_out, ws, K_out=None, V_out=None, pos_out=None, weight_out=None,
                   stream=None):
    """Without K_out, V_out, pos_out, weight_out [B, H_kv, out_capacity(, d)]: in place."""
    dev, sd = _device("K_cache", K_cache), _STORAGE[c.dtype]
    B, Hk, d, cap = c.batch, c.n_kv_heads, c.head_dim, c.capacity
    cache, slots = (B, Hk, cap, d), (B, Hk, cap)
    kc, vc = _whole("K_cache", K_cache, cache, sd, dev), _whole("V_cache", V_cache, cache, sd, dev)
    sp, w = _whole("slot_pos", slot_pos, slots, _I32, dev), _whole("weight", weight, slots, _F32, dev)
    ko, vo, po, wo = kc, vc, sp, w
    if K_out is not None or V_out is not None or pos_out is not None or weight_out is not None:
        if K_out is None or V_out is None or pos_out is None or weight_out is None:
            raise ValueError("K_out, V_out, pos_out and weight_out are given together")
        cap = K_out.shape[2] if K_out.dim() == 4 else cap
        cache, slots = (B, Hk, cap, d), (B, Hk, cap)
        ko, vo = _whole("K_out", K_out, cache, sd, dev), _whole("V_out", V_out, cache, sd, dev)
        po, wo = _whole("pos_out", pos_out, slots, _I32, dev), _whole("weight_out", weight_out, slots, _F32, dev)
    _call(load_library().tc_cache_evict, dev, stream, c, _whole("lens", lens, (B,), _I32, dev), kc, vc, sp, w, ko, vo, po, wo, cap,
          _whole("len_out", len_out, (B,), _I32, dev), _whole("ws", ws, (ws.numel(),), _U8, dev), ws.numel())
