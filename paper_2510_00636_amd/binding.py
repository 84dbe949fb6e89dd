"""ctypes binding of include/ea.h and include/ea_profile.h -- same names, argument marshalling only.

Tensor arguments are torch CUDA tensors (or anything with .data_ptr()); `stream` is a
torch.cuda.Stream, a raw hipStream_t integer, or None for torch's current stream."""
import ctypes
import os

EA_F32, EA_BF16, EA_FP8_E4M3 = 0, 1, 2
_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class EaError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__("%s: %s (status %d)" % (where, status_string(code), code))


class EaParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("rope_layout", ctypes.c_int32),
                ("q_is_rotated", ctypes.c_int32), ("cov_ddof", ctypes.c_int32),
                ("horizon_T", ctypes.c_int32), ("epsilon", ctypes.c_float)]


class EaPaged(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("block_size", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("num_blocks", ctypes.c_int64)]


class EaNewRows(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64), ("n_tokens", ctypes.c_int64),
                ("pos", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p)]


class EaStep(ctypes.Structure):
    _fields_ = [("cu_tokens", ctypes.c_void_p), ("n_tokens", ctypes.c_int64), ("max_new", ctypes.c_int64),
                ("q_stride", ctypes.c_int64)]


EA_MXFP8, EA_MXFP4 = 0, 1


class EaMx(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("format", ctypes.c_int32)]


class EaTree(ctypes.Structure):
    _fields_ = [("sees", ctypes.c_void_p), ("words", ctypes.c_int32)]


def lib_path():
    """In-tree libea.so; the environment variable EA_LIBRARY names another build of it."""
    return os.environ.get("EA_LIBRARY") or os.path.join(_HERE, "libea.so")


def load_library():
    """Loads libea.so (built in-tree by paper_2510_00636_amd.build).  Raises if it is absent:
    there is deliberately no fallback implementation."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError("libea.so not found at %s -- run `python -m paper_2510_00636_amd.build` "
                           "(or __graft_entry__.build()) first" % path)
    lib = ctypes.CDLL(path)
    P, VP, I64, SZ = ctypes.POINTER(EaParams), ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    lib.ea_workspace_bytes.restype = SZ
    lib.ea_workspace_bytes.argtypes = [P, I64, I64]
    lib.ea_query_stats.restype = ctypes.c_int
    lib.ea_query_stats.argtypes = [P, VP, I64, I64, VP, I64, VP, VP, VP, SZ, VP]
    lib.ea_query_stats_hidden.restype = ctypes.c_int
    lib.ea_query_stats_hidden.argtypes = [P, VP, VP, I64, I64, VP, I64, VP, VP, VP, SZ, VP]
    lib.ea_score.restype = ctypes.c_int
    lib.ea_score.argtypes = [P, VP, VP, I64, I64, VP, VP, VP, VP, SZ, VP]
    lib.ea_select.restype = ctypes.c_int
    lib.ea_select.argtypes = [P, VP, I64, I64, VP, VP, SZ, VP]
    lib.ea_wo_gram.restype = ctypes.c_int
    lib.ea_wo_gram.argtypes = [P, VP, I64, VP, VP]
    lib.ea_value_norms_wo.restype = ctypes.c_int
    lib.ea_value_norms_wo.argtypes = [P, VP, I64, I64, VP, VP, VP, SZ, VP]
    lib.ea_score_wo.restype = ctypes.c_int
    lib.ea_score_wo.argtypes = [P, VP, VP, I64, I64, VP, VP, VP, VP, VP, SZ, VP]
    lib.ea_select_static.restype = ctypes.c_int
    lib.ea_select_static.argtypes = [P, VP, I64, I64, VP, VP]
    lib.ea_compact.restype = ctypes.c_int
    lib.ea_compact.argtypes = [P, VP, VP, I64, I64, VP, I64, VP, VP, VP, SZ, VP]
    lib.ea_compress_layer.restype = ctypes.c_int
    lib.ea_compress_layer.argtypes = [P, VP, I64, I64, VP, I64, VP, VP, I64, I64, I64, VP, VP, VP, SZ, VP]
    lib.ea_select_adaptive.restype = ctypes.c_int
    lib.ea_select_adaptive.argtypes = [P, VP, I64, I64, I64, VP, VP, VP, SZ, VP]
    lib.ea_compress_layer_adaptive.restype = ctypes.c_int
    lib.ea_compress_layer_adaptive.argtypes = [P, VP, I64, I64, VP, I64, VP, VP, I64, I64, I64, I64, VP, VP, VP, VP,
                                               SZ, VP]
    lib.ea_compact_ragged.restype = ctypes.c_int
    lib.ea_compact_ragged.argtypes = [P, VP, VP, I64, I64, VP, VP, VP, SZ, VP]
    lib.ea_score_baseline.restype = ctypes.c_int
    lib.ea_score_baseline.argtypes = [P, ctypes.c_int32, VP, I64, I64, I64, VP, VP, SZ, VP]
    lib.ea_compact_unordered.restype = ctypes.c_int
    lib.ea_compact_unordered.argtypes = [P, VP, VP, I64, I64, VP, I64, VP, VP]
    lib.ea_compress_layer_unordered.restype = ctypes.c_int
    lib.ea_compress_layer_unordered.argtypes = [P, VP, I64, I64, VP, I64, VP, VP, I64, I64, I64, VP, VP, VP, VP, SZ, VP]
    PG = ctypes.POINTER(EaPaged)
    lib.ea_score_paged.restype = ctypes.c_int
    lib.ea_score_paged.argtypes = [P, VP, VP, PG, I64, VP, VP, VP, VP, SZ, VP]
    lib.ea_compact_paged.restype = ctypes.c_int
    lib.ea_compact_paged.argtypes = [P, VP, VP, PG, I64, VP, I64, ctypes.c_int32, VP, VP, SZ, VP]
    lib.ea_compress_layer_paged.restype = ctypes.c_int
    lib.ea_compress_layer_paged.argtypes = [P, VP, I64, I64, VP, I64, VP, VP, PG, I64, I64, ctypes.c_int32,
                                            VP, VP, VP, VP, SZ, VP]
    lib.ea_score_fp8.restype = ctypes.c_int
    lib.ea_score_fp8.argtypes = [P, VP, VP, VP, VP, I64, I64, VP, VP, VP, VP, SZ, VP]
    lib.ea_compress_layer_fp8.restype = ctypes.c_int
    lib.ea_compress_layer_fp8.argtypes = [P, VP, I64, I64, VP, I64, VP, VP, VP, VP, I64, I64, I64, ctypes.c_int32,
                                          VP, VP, VP, VP, SZ, VP]
    NR, ST = ctypes.POINTER(EaNewRows), ctypes.POINTER(EaStep)
    lib.ea_block_tables.restype = ctypes.c_int
    lib.ea_block_tables.argtypes = [P, PG, VP, VP, VP, VP, VP, VP, VP, I64, VP, VP, VP, VP]
    lib.ea_append_paged.restype = ctypes.c_int
    lib.ea_append_paged.argtypes = [P, NR, VP, VP, VP, PG, VP, VP]
    lib.ea_append.restype = ctypes.c_int
    lib.ea_append.argtypes = [P, NR, VP, VP, VP, VP, I64, VP, VP]
    lib.ea_append_fp8.restype = ctypes.c_int
    lib.ea_append_fp8.argtypes = [P, NR, VP, VP, VP, VP, VP, VP, I64, VP, VP]
    lib.ea_attend_workspace_bytes.restype = SZ
    lib.ea_attend_workspace_bytes.argtypes = [P, ST, I64]
    lib.ea_attend.restype = ctypes.c_int
    lib.ea_attend.argtypes = [P, VP, ST, VP, VP, VP, I64, I64, VP, VP, VP, SZ, VP]
    lib.ea_attend_paged.restype = ctypes.c_int
    lib.ea_attend_paged.argtypes = [P, VP, ST, VP, VP, PG, VP, I64, VP, VP, VP, SZ, VP]
    lib.ea_attend_fp8.restype = ctypes.c_int
    lib.ea_attend_fp8.argtypes = [P, VP, ST, VP, VP, VP, VP, VP, I64, I64, VP, VP, VP, SZ, VP]
    MX, TR = ctypes.POINTER(EaMx), ctypes.POINTER(EaTree)
    for name, args in (("append_mx", [P, NR, VP, MX, PG, VP, VP]), ("read_mx", [P, MX, PG, VP, I64, I64, VP, VP, VP]),
                       ("attend_mx", [P, VP, ST, MX, PG, VP, I64, VP, VP, VP, SZ, VP]),
                       ("tree_masks", [P, ST, VP, TR, VP, VP, VP]), ("tree_accept", [P, ST, VP, VP, VP, VP, VP, VP, VP]),
                       ("attend_tree", [P, VP, ST, TR, VP, VP, VP, I64, I64, VP, VP, VP, SZ, VP]),
                       ("attend_tree_fp8", [P, VP, ST, TR, VP, VP, VP, VP, VP, I64, I64, VP, VP, VP, SZ, VP]),
                       ("attend_tree_paged", [P, VP, ST, TR, VP, VP, PG, VP, I64, VP, VP, VP, SZ, VP]),
                       ("attend_tree_mx", [P, VP, ST, TR, MX, PG, VP, I64, VP, VP, VP, SZ, VP]),
                       ("keep_path", [P, ST, VP, VP, VP, VP, VP, I64, VP, VP]),
                       ("keep_path_paged", [P, ST, VP, VP, VP, VP, PG, VP, VP, VP, VP]),
                       ("keep_path_mx", [P, ST, VP, VP, MX, PG, VP, VP, VP, VP])):
        f = getattr(lib, "ea_" + name)
        f.restype, f.argtypes = ctypes.c_int, args
    lib.ea_compress_layer_timed.restype = ctypes.c_int
    lib.ea_compress_layer_timed.argtypes = [P, VP, I64, I64, VP, I64, VP, VP, I64, I64, I64, VP, SZ, VP,
                                            ctypes.POINTER(ctypes.c_float)]
    lib.ea_debug_status.restype = ctypes.c_int
    lib.ea_debug_status.argtypes = [P, I64, I64, VP, SZ, VP, ctypes.POINTER(ctypes.c_uint32)]
    lib.ea_n_keep.restype = I64
    lib.ea_n_keep.argtypes = [I64, ctypes.c_double]
    lib.ea_status_string.restype = ctypes.c_char_p
    lib.ea_status_string.argtypes = [ctypes.c_int]
    _LIB = lib
    return lib


def make_params(batch, n_q_heads, n_kv_heads, head_dim, dtype, rope_layout=0, q_is_rotated=1,
                cov_ddof=0, horizon_T=512, epsilon=0.02):
    return EaParams(batch, n_q_heads, n_kv_heads, head_dim, dtype, rope_layout, q_is_rotated,
                    cov_ddof, horizon_T, epsilon)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return ctypes.c_void_p(t)
    return ctypes.c_void_p(t.data_ptr())


def _nbytes(t):
    return t.numel() * t.element_size()


def _stream(s):
    if s is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(s, int):
        return ctypes.c_void_p(s)
    return ctypes.c_void_p(s.cuda_stream)


def _check(code, where):
    if code != 0:
        raise EaError(code, where)


def status_string(code):
    return load_library().ea_status_string(int(code)).decode()


def n_keep(n, ratio):
    return int(load_library().ea_n_keep(int(n), float(ratio)))


def workspace_bytes(p, n, window):
    return int(load_library().ea_workspace_bytes(ctypes.byref(p), int(n), int(window)))


def query_stats(p, q_win, window, q_pos0, inv_freq, t_next, mu, sigma, ws, stream=None):
    _check(load_library().ea_query_stats(ctypes.byref(p), _ptr(q_win), int(window), int(q_pos0),
                                         _ptr(inv_freq), int(t_next), _ptr(mu), _ptr(sigma),
                                         _ptr(ws), _nbytes(ws), _stream(stream)), "ea_query_stats")


def query_stats_hidden(p, hidden, w_q, d_model, window, inv_freq, t_next, mu, sigma, ws, stream=None):
    _check(load_library().ea_query_stats_hidden(ctypes.byref(p), _ptr(hidden), _ptr(w_q), int(d_model),
                                                int(window), _ptr(inv_freq), int(t_next), _ptr(mu),
                                                _ptr(sigma), _ptr(ws), _nbytes(ws), _stream(stream)),
           "ea_query_stats_hidden")


def wo_gram(p, w_o, d_model, gram, stream=None):
    _check(load_library().ea_wo_gram(ctypes.byref(p), _ptr(w_o), int(d_model), _ptr(gram), _stream(stream)),
           "ea_wo_gram")


def value_norms_wo(p, v, n, n_cap, gram, wnorm, ws, stream=None):
    _check(load_library().ea_value_norms_wo(ctypes.byref(p), _ptr(v), int(n), int(n_cap), _ptr(gram),
                                            _ptr(wnorm), _ptr(ws), _nbytes(ws), _stream(stream)),
           "ea_value_norms_wo")


def score_wo(p, k, v, n, n_cap, mu, sigma, wnorm, scores, ws, stream=None):
    _check(load_library().ea_score_wo(ctypes.byref(p), _ptr(k), _ptr(v), int(n), int(n_cap), _ptr(mu),
                                      _ptr(sigma), _ptr(wnorm), _ptr(scores), _ptr(ws), _nbytes(ws),
                                      _stream(stream)), "ea_score_wo")


def score(p, k, v, n, n_cap, mu, sigma, scores, ws, stream=None):
    _check(load_library().ea_score(ctypes.byref(p), _ptr(k), _ptr(v), int(n), int(n_cap), _ptr(mu),
                                   _ptr(sigma), _ptr(scores), _ptr(ws), _nbytes(ws),
                                   _stream(stream)), "ea_score")


def select(p, scores, n, n_keep_, idx, ws, stream=None):
    _check(load_library().ea_select(ctypes.byref(p), _ptr(scores), int(n), int(n_keep_), _ptr(idx),
                                    _ptr(ws), _nbytes(ws), _stream(stream)), "ea_select")


def select_static(p, scores, n, n_keep_, idx, stream=None):
    _check(load_library().ea_select_static(ctypes.byref(p), _ptr(scores), int(n), int(n_keep_),
                                           _ptr(idx), _stream(stream)), "ea_select_static")


def compact(p, k, v, n, n_cap, idx, n_keep_, k_out, v_out, ws, stream=None):
    _check(load_library().ea_compact(ctypes.byref(p), _ptr(k), _ptr(v), int(n), int(n_cap),
                                     _ptr(idx), int(n_keep_), _ptr(k_out), _ptr(v_out), _ptr(ws),
                                     _nbytes(ws), _stream(stream)), "ea_compact")


def compress_layer(p, q_win, window, q_pos0, inv_freq, t_next, k, v, n, n_cap, n_keep_,
                   scores_out, idx_out, ws, stream=None):
    _check(load_library().ea_compress_layer(ctypes.byref(p), _ptr(q_win), int(window), int(q_pos0),
                                            _ptr(inv_freq), int(t_next), _ptr(k), _ptr(v), int(n),
                                            int(n_cap), int(n_keep_), _ptr(scores_out),
                                            _ptr(idx_out), _ptr(ws), _nbytes(ws), _stream(stream)),
           "ea_compress_layer")


def select_adaptive(p, scores, n, n_keep_, floor, idx, lengths, ws, stream=None):
    _check(load_library().ea_select_adaptive(ctypes.byref(p), _ptr(scores), int(n), int(n_keep_), int(floor),
                                             _ptr(idx), _ptr(lengths), _ptr(ws), _nbytes(ws),
                                             _stream(stream)), "ea_select_adaptive")


def compress_layer_adaptive(p, q_win, window, q_pos0, inv_freq, t_next, k, v, n, n_cap, n_keep_, floor,
                            scores_out, idx_out, lengths_out, ws, stream=None):
    _check(load_library().ea_compress_layer_adaptive(ctypes.byref(p), _ptr(q_win), int(window), int(q_pos0),
                                                     _ptr(inv_freq), int(t_next), _ptr(k), _ptr(v), int(n),
                                                     int(n_cap), int(n_keep_), int(floor), _ptr(scores_out),
                                                     _ptr(idx_out), _ptr(lengths_out), _ptr(ws), _nbytes(ws),
                                                     _stream(stream)), "ea_compress_layer_adaptive")


def compact_ragged(p, k, v, n, n_cap, idx, lengths, ws, stream=None):
    _check(load_library().ea_compact_ragged(ctypes.byref(p), _ptr(k), _ptr(v), int(n), int(n_cap), _ptr(idx),
                                            _ptr(lengths), _ptr(ws), _nbytes(ws), _stream(stream)),
           "ea_compact_ragged")


SCORER_KNORM, SCORER_STREAMING, SCORER_KEYDIFF = 0, 1, 2


def score_baseline(p, scorer, k, n, n_cap, n_sink, scores, ws, stream=None):
    _check(load_library().ea_score_baseline(ctypes.byref(p), int(scorer), _ptr(k), int(n), int(n_cap),
                                            int(n_sink), _ptr(scores), _ptr(ws), _nbytes(ws),
                                            _stream(stream)), "ea_score_baseline")


def compact_unordered(p, k, v, n, n_cap, idx, n_keep_, perm_out=None, stream=None):
    _check(load_library().ea_compact_unordered(ctypes.byref(p), _ptr(k), _ptr(v), int(n), int(n_cap),
                                               _ptr(idx), int(n_keep_), _ptr(perm_out), _stream(stream)),
           "ea_compact_unordered")


def compress_layer_unordered(p, q_win, window, q_pos0, inv_freq, t_next, k, v, n, n_cap, n_keep_,
                             scores_out, idx_out, perm_out, ws, stream=None):
    _check(load_library().ea_compress_layer_unordered(ctypes.byref(p), _ptr(q_win), int(window),
                                                      int(q_pos0), _ptr(inv_freq), int(t_next), _ptr(k),
                                                      _ptr(v), int(n), int(n_cap), int(n_keep_),
                                                      _ptr(scores_out), _ptr(idx_out), _ptr(perm_out),
                                                      _ptr(ws), _nbytes(ws), _stream(stream)),
           "ea_compress_layer_unordered")


def make_paged(block_table, block_size, num_blocks):
    """ea_paged for a block table tensor [B, max_blocks] int32 on the device."""
    return EaPaged(block_table.data_ptr(), int(block_size), int(block_table.shape[-1]), int(num_blocks))


def score_paged(p, k_pool, v_pool, pg, n, mu, sigma, scores, ws, stream=None):
    _check(load_library().ea_score_paged(ctypes.byref(p), _ptr(k_pool), _ptr(v_pool), ctypes.byref(pg), int(n),
                                         _ptr(mu), _ptr(sigma), _ptr(scores), _ptr(ws), _nbytes(ws),
                                         _stream(stream)), "ea_score_paged")


def compact_paged(p, k_pool, v_pool, pg, n, idx, n_keep_, order_free, perm_out, ws, stream=None):
    _check(load_library().ea_compact_paged(ctypes.byref(p), _ptr(k_pool), _ptr(v_pool), ctypes.byref(pg), int(n),
                                           _ptr(idx), int(n_keep_), int(order_free), _ptr(perm_out), _ptr(ws),
                                           _nbytes(ws), _stream(stream)), "ea_compact_paged")


def compress_layer_paged(p, q_win, window, q_pos0, inv_freq, t_next, k_pool, v_pool, pg, n, n_keep_, order_free,
                         scores_out, idx_out, perm_out, ws, stream=None):
    _check(load_library().ea_compress_layer_paged(ctypes.byref(p), _ptr(q_win), int(window), int(q_pos0),
                                                  _ptr(inv_freq), int(t_next), _ptr(k_pool), _ptr(v_pool),
                                                  ctypes.byref(pg), int(n), int(n_keep_), int(order_free),
                                                  _ptr(scores_out), _ptr(idx_out), _ptr(perm_out), _ptr(ws),
                                                  _nbytes(ws), _stream(stream)), "ea_compress_layer_paged")


def score_fp8(p, k8, v8, k_scale, v_scale, n, n_cap, mu, sigma, scores, ws, stream=None):
    _check(load_library().ea_score_fp8(ctypes.byref(p), _ptr(k8), _ptr(v8), _ptr(k_scale), _ptr(v_scale), int(n),
                                       int(n_cap), _ptr(mu), _ptr(sigma), _ptr(scores), _ptr(ws), _nbytes(ws),
                                       _stream(stream)), "ea_score_fp8")


def compress_layer_fp8(p, q_win, window, q_pos0, inv_freq, t_next, k8, v8, k_scale, v_scale, n, n_cap, n_keep_,
                       order_free, scores_out, idx_out, perm_out, ws, stream=None):
    _check(load_library().ea_compress_layer_fp8(ctypes.byref(p), _ptr(q_win), int(window), int(q_pos0),
                                                _ptr(inv_freq), int(t_next), _ptr(k8), _ptr(v8), _ptr(k_scale),
                                                _ptr(v_scale), int(n), int(n_cap), int(n_keep_), int(order_free),
                                                _ptr(scores_out), _ptr(idx_out), _ptr(perm_out), _ptr(ws),
                                                _nbytes(ws), _stream(stream)), "ea_compress_layer_fp8")


def _addr(t):
    """As _ptr, without an object of its own: what ctypes takes for a void*."""
    return t if t is None or isinstance(t, int) else t.data_ptr()


_torch_c = None


def _now(s):
    """The stream's handle.  A step's calls are short next to what the host spends on one, so torch's current stream is asked for
    by the call that its own kernels use (2 us less than a Stream object)."""
    if s is None:
        global _torch_c
        if _torch_c is None:
            import torch
            _torch_c = torch._C
        return _torch_c._cuda_getCurrentRawStream(_torch_c._cuda_getDevice())
    return s if isinstance(s, int) else s.cuda_stream


def block_tables(p, pg, len_old, len_new, free_list, free_in, len_out, free_out, cu_tokens, n_tokens=0, slots=None, pos=None,
                 seen=None, stream=None):
    """Writes the block table that pg points at, too."""
    _check(load_library().ea_block_tables(p, pg, _addr(len_old), _addr(len_new), _addr(free_list), _addr(free_in), _addr(len_out),
                                          _addr(free_out), _addr(cu_tokens), int(n_tokens), _addr(slots), _addr(pos), _addr(seen),
                                          _now(stream)), "ea_block_tables")


def _token_stride(t):
    """Elements from one token to the next of t [n_tokens, heads, d]; a token's heads have to stand together, and no two tokens in
    one place (0 would stand for dense rows, more of them than there are)."""
    if t.dim() != 3 or t.stride(-1) != 1 or (t.shape[-2] > 1 and t.stride(-2) != t.shape[-1]):
        raise ValueError("rows are [tokens, heads, d], the heads of a token contiguous")
    if t.shape[0] < 2:
        return 0
    if t.stride(0) < t.shape[-2] * t.shape[-1]:
        raise ValueError("tokens must not share memory")
    return t.stride(0)


def make_new_rows(q, k, v, pos=None, inv_freq=None):
    """ea_new_rows for tensors q (or None) [n_tokens, Hq, d], k, v [n_tokens, Hkv, d]; views into one projection's rows will do.
    pos int32 [n_tokens or more], inv_freq float64 [d / 2]."""
    def ptr(t):
        return None if t is None else t.data_ptr()
    strides = [0 if t is None else _token_stride(t) for t in (q, k, v)]
    # the library reads as many rows of each as k has
    if v.shape != k.shape or (q is not None and (q.shape[0], q.shape[2]) != (k.shape[0], k.shape[2])):
        raise ValueError("q, k and v must have the same tokens and channels, k and v the same heads")
    if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise ValueError("q, k and v must have one type")
    if inv_freq is not None:
        if pos is None or pos.numel() < k.shape[0] or pos.element_size() != 4 or not pos.is_contiguous():
            raise ValueError("pos must be int32, one for each token")
        if inv_freq.numel() != k.shape[2] // 2 or inv_freq.element_size() != 8 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be float64 [d / 2]")
    r = EaNewRows(ptr(q), ptr(k), ptr(v), *strides, k.shape[0], ptr(pos), ptr(inv_freq))
    r.tensors = (q, k, v, pos, inv_freq)      # alive as long as the addresses are kept
    return r


def append_paged(p, rows, slots, k_pool, v_pool, pg, q_out=None, stream=None):
    _check(load_library().ea_append_paged(p, rows, _addr(slots), _addr(k_pool), _addr(v_pool),
                                          pg, _addr(q_out), _now(stream)), "ea_append_paged")


def append(p, rows, cu_tokens, lengths, k, v, n_cap, q_out=None, stream=None):
    _check(load_library().ea_append(p, rows, _addr(cu_tokens), _addr(lengths), _addr(k), _addr(v),
                                    int(n_cap), _addr(q_out), _now(stream)), "ea_append")


def append_fp8(p, rows, cu_tokens, lengths, k8, v8, k_scale, v_scale, n_cap, q_out=None, stream=None):
    _check(load_library().ea_append_fp8(p, rows, _addr(cu_tokens), _addr(lengths), _addr(k8), _addr(v8),
                                        _addr(k_scale), _addr(v_scale), int(n_cap), _addr(q_out), _now(stream)), "ea_append_fp8")


def make_step(cu_tokens, n_tokens, max_new, q_stride=0):
    """ea_step for a tensor of prefix sums [B + 1] int32 on the device."""
    s = EaStep(cu_tokens.data_ptr(), int(n_tokens), int(max_new), int(q_stride))
    s.tensors = (cu_tokens,)
    return s


def attend_workspace_bytes(p, step, n):
    return int(load_library().ea_attend_workspace_bytes(p, step, int(n)))


def attend(p, q, step, k, v, lengths, n, n_cap, out, lse, ws, stream=None):
    _check(load_library().ea_attend(p, _addr(q), step, _addr(k), _addr(v), _addr(lengths), int(n),
                                    int(n_cap), _addr(out), _addr(lse), _addr(ws), _nbytes(ws), _now(stream)), "ea_attend")


def attend_paged(p, q, step, k_pool, v_pool, pg, lengths, n, out, lse, ws, stream=None):
    _check(load_library().ea_attend_paged(p, _addr(q), step, _addr(k_pool), _addr(v_pool),
                                          pg, _addr(lengths), int(n), _addr(out), _addr(lse), _addr(ws), _nbytes(ws),
                                          _now(stream)), "ea_attend_paged")


def attend_fp8(p, q, step, k8, v8, k_scale, v_scale, lengths, n, n_cap, out, lse, ws, stream=None):
    _check(load_library().ea_attend_fp8(p, _addr(q), step, _addr(k8), _addr(v8), _addr(k_scale),
                                        _addr(v_scale), _addr(lengths), int(n), int(n_cap), _addr(out), _addr(lse), _addr(ws),
                                        _nbytes(ws), _now(stream)), "ea_attend_fp8")


def make_mx(k, v, k_scale, v_scale, fmt):
    """ea_mx for pools [num_blocks, Hkv, block_size, d (EA_MXFP4: d / 2)] of bytes and their scales [num_blocks, Hkv, block_size, d / 32]."""
    for x, s in ((k, k_scale), (v, v_scale)):
        if x.element_size() != 1 or s.element_size() != 1 or not x.is_contiguous() or not s.is_contiguous():
            raise ValueError("elements and scales are contiguous tensors of bytes")
        if x.shape[:-1] != s.shape[:-1] or x.shape[-1] * (2 if fmt == EA_MXFP4 else 1) != s.shape[-1] * 32:
            raise ValueError("a row has one scale for 32 channels")
    if k.shape != v.shape:
        raise ValueError("k and v must have the same shape")
    m = EaMx(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), int(fmt))
    m.tensors = (k, v, k_scale, v_scale)
    return m


def append_mx(p, rows, slots, mx, pg, q_out=None, stream=None):
    _check(load_library().ea_append_mx(p, rows, _addr(slots), mx, pg, _addr(q_out), _now(stream)), "ea_append_mx")


def read_mx(p, mx, pg, lengths, n, n_cap, k_out, v_out, stream=None):
    _check(load_library().ea_read_mx(p, mx, pg, _addr(lengths), int(n), int(n_cap), _addr(k_out), _addr(v_out), _now(stream)), "ea_read_mx")


def attend_mx(p, q, step, mx, pg, lengths, n, out, lse, ws, stream=None):
    _check(load_library().ea_attend_mx(p, _addr(q), step, mx, pg, _addr(lengths), int(n), _addr(out), _addr(lse), _addr(ws),
                                       _nbytes(ws), _now(stream)), "ea_attend_mx")


def make_tree(sees):
    """ea_tree for a tensor of masks [n_tokens, words] int64 on the device."""
    if sees.dim() != 2 or sees.element_size() != 8 or sees.is_floating_point() or sees.is_complex() or not sees.is_contiguous():
        raise ValueError("masks are [tokens, words] of 64 bits, contiguous")
    t = EaTree(sees.data_ptr(), int(sees.shape[1]))
    t.tensors = (sees,)
    return t


def tree_masks(p, step, parents, tree, pos=None, seen=None, stream=None):
    """Writes the masks that tree points at, too."""
    _check(load_library().ea_tree_masks(p, step, _addr(parents), tree, _addr(seen), _addr(pos), _now(stream)), "ea_tree_masks")


def tree_accept(p, step, tokens, parents, target, path, n_path, next_token, stream=None):
    _check(load_library().ea_tree_accept(p, step, _addr(tokens), _addr(parents), _addr(target), _addr(path), _addr(n_path),
                                         _addr(next_token), _now(stream)), "ea_tree_accept")


def attend_tree(p, q, step, tree, k, v, lengths, n, n_cap, out, lse, ws, stream=None):
    _check(load_library().ea_attend_tree(p, _addr(q), step, tree, _addr(k), _addr(v), _addr(lengths), int(n), int(n_cap), _addr(out),
                                         _addr(lse), _addr(ws), _nbytes(ws), _now(stream)), "ea_attend_tree")


def attend_tree_fp8(p, q, step, tree, k8, v8, k_scale, v_scale, lengths, n, n_cap, out, lse, ws, stream=None):
    _check(load_library().ea_attend_tree_fp8(p, _addr(q), step, tree, _addr(k8), _addr(v8), _addr(k_scale), _addr(v_scale),
                                             _addr(lengths), int(n), int(n_cap), _addr(out), _addr(lse), _addr(ws), _nbytes(ws),
                                             _now(stream)), "ea_attend_tree_fp8")


def attend_tree_paged(p, q, step, tree, k_pool, v_pool, pg, lengths, n, out, lse, ws, stream=None):
    _check(load_library().ea_attend_tree_paged(p, _addr(q), step, tree, _addr(k_pool), _addr(v_pool), pg, _addr(lengths), int(n),
                                               _addr(out), _addr(lse), _addr(ws), _nbytes(ws), _now(stream)), "ea_attend_tree_paged")


def attend_tree_mx(p, q, step, tree, mx, pg, lengths, n, out, lse, ws, stream=None):
    _check(load_library().ea_attend_tree_mx(p, _addr(q), step, tree, mx, pg, _addr(lengths), int(n), _addr(out), _addr(lse),
                                            _addr(ws), _nbytes(ws), _now(stream)), "ea_attend_tree_mx")


def keep_path(p, step, path, n_path, k, v, lengths, n_cap, len_out, stream=None):
    _check(load_library().ea_keep_path(p, step, _addr(path), _addr(n_path), _addr(k), _addr(v), _addr(lengths), int(n_cap),
                                       _addr(len_out), _now(stream)), "ea_keep_path")


def keep_path_paged(p, step, path, n_path, k_pool, v_pool, pg, lengths, len_out, slots=None, stream=None):
    _check(load_library().ea_keep_path_paged(p, step, _addr(path), _addr(n_path), _addr(k_pool), _addr(v_pool), pg, _addr(slots),
                                             _addr(lengths), _addr(len_out), _now(stream)), "ea_keep_path_paged")


def keep_path_mx(p, step, path, n_path, mx, pg, lengths, len_out, slots=None, stream=None):
    _check(load_library().ea_keep_path_mx(p, step, _addr(path), _addr(n_path), mx, pg, _addr(slots), _addr(lengths), _addr(len_out),
                                          _now(stream)), "ea_keep_path_mx")


N_STAGES = 6
STAGE_NAMES = ("stats", "prep", "score_a", "score_b", "select", "compact")


def compress_layer_timed(p, q_win, window, q_pos0, inv_freq, t_next, k, v, n, n_cap, n_keep_, ws,
                         stream=None):
    """Profiling variant: returns the six stage times in milliseconds (host floats)."""
    ms = (ctypes.c_float * N_STAGES)()
    _check(load_library().ea_compress_layer_timed(ctypes.byref(p), _ptr(q_win), int(window),
                                                  int(q_pos0), _ptr(inv_freq), int(t_next), _ptr(k),
                                                  _ptr(v), int(n), int(n_cap), int(n_keep_), _ptr(ws),
                                                  _nbytes(ws), _stream(stream), ms),
           "ea_compress_layer_timed")
    return list(ms)


STATUS_BAD_SCORE, STATUS_COMPACT_WAIT, STATUS_BAD_INDEX = 1, 2, 4


def debug_status(p, n, window, ws, stream=None):
    """Debugging aid (blocks): the status bits the kernels left in the workspace."""
    word = ctypes.c_uint32(0)
    _check(load_library().ea_debug_status(ctypes.byref(p), int(n), int(window), _ptr(ws), _nbytes(ws),
                                          _stream(stream), ctypes.byref(word)), "ea_debug_status")
    return int(word.value)
