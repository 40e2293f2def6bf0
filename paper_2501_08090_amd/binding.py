"""Thin ctypes binding of libchiron.so (include/chiron.h, include/chiron_ops.h).

Argument marshalling only: every function takes torch tensors that already live on the
GPU (torch supplies device memory and streams), checks dtype/contiguity, and passes raw
pointers through the C ABI.  No step of the decode path runs in Python, and there is no
fallback: if the library has not been built, loading raises.
"""
import ctypes as C
import os
from operator import index

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("CHIRON_LIB", os.path.join(_HERE, "libchiron.so"))

CHIRON_BF16 = 1
CHIRON_F32 = 2
ERRORS = {0: "OK", -1: "INVALID_ARG", -2: "SHAPE", -3: "BATCH_TOO_LARGE", -4: "BLOCK_TABLE", -5: "OOM", -6: "HIP", -7: "TOKEN"}

# every symbol the headers declare (tests check that the library exports all of them)
SYMBOLS = [
    "chiron_model_create", "chiron_model_load_layer", "chiron_model_load_head", "chiron_model_destroy",
    "chiron_kv_block_bytes", "chiron_kv_pool_create", "chiron_kv_pool_destroy", "chiron_append_kv", "chiron_gather_kv",
    "chiron_kv_swap_out", "chiron_kv_swap_in",
    "chiron_decode_step", "chiron_decode_step_multi", "chiron_validate_step_inputs", "chiron_check_step_inputs_host",
    "chiron_validate_step_inputs_multi", "chiron_check_step_inputs_host_multi", "chiron_step_latency_profile",
    "chiron_last_error", "chiron_kernel_timing_begin", "chiron_kernel_timing_end", "chiron_local_autoscale_step",
    "chiron_op_rmsnorm", "chiron_linear_create", "chiron_linear_destroy", "chiron_op_linear", "chiron_linear_create_gate_up", "chiron_op_gate_up_swiglu", "chiron_op_swiglu_ffn",
    "chiron_op_rope", "chiron_op_rope_noalloc", "chiron_op_paged_attention", "chiron_set_tuning",
    "chiron_append_kv_rope", "chiron_kv_index_bytes", "chiron_kv_index_create", "chiron_kv_index_destroy", "chiron_kv_index_update",
    "chiron_op_rope_table", "chiron_op_select_pages", "chiron_op_sparse_attention", "chiron_verify_workspace_bytes",
    "chiron_op_verify_drafts", "chiron_linear4_create", "chiron_linear4_destroy", "chiron_op_linear4",
    "chiron_linear4_workspace_bytes",
]


class ChironError(RuntimeError):
    def __init__(self, code, text):
        super().__init__("chiron: %s (%d): %s" % (ERRORS.get(code, "?"), code, text))
        self.code = code


class ModelConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab")] + [
        ("rope_base", C.c_float), ("rms_eps", C.c_float), ("dtype", C.c_int32), ("max_batch", C.c_int32),
        ("max_blocks_per_seq", C.c_int32)]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")]


class NewRows(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "k", "v")] + [(n, C.c_int64) for n in ("q_stride", "k_stride", "v_stride")] + [
        ("dtype", C.c_int32), ("n_q_heads", C.c_int32)] + [(n, C.c_void_p) for n in ("cos", "sin", "q_out")]


class DraftBatch(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("draft_logits", C.c_void_p), ("logits_stride", C.c_int64), ("draft_stride", C.c_int64)] + [
        (n, C.c_void_p) for n in ("tokens", "draft_lens", "uniforms", "noise", "temperature")]


class ProfilePoint(C.Structure):
    _fields_ = [("batch", C.c_int32), ("lat_ms_median", C.c_double), ("lat_ms_p99", C.c_double),
                ("lat_ms_mean", C.c_double), ("tokens_per_s", C.c_double)]


_lib = None

# Entry points that a serving loop calls again and again, with their argument types (p: pointer or stream, i: int32, l: int64): their
# arguments go in as plain numbers, without a ctypes object for each (5.2 -> 2.6 us of Python a call).  What a caller hands in as a number
# goes through index() first: no whole number is a TypeError, where ctypes would raise an ArgumentError, which is none.
_HOT = {"chiron_decode_step": "pppppipp", "chiron_decode_step_multi": "pppppiipp", "chiron_append_kv": "pipppipplp",
        "chiron_gather_kv": "pipippp", "chiron_kv_swap_out": "ppipp", "chiron_kv_swap_in": "ppipp", "chiron_op_linear": "ppipip",
        "chiron_op_gate_up_swiglu": "ppipp", "chiron_op_swiglu_ffn": "pppipip", "chiron_op_paged_attention": "ppipppipp",
        "chiron_append_kv_rope": "ppippippiip", "chiron_kv_index_update": "ppiipippiip", "chiron_op_select_pages": "pppippppiiiippp",
        "chiron_op_sparse_attention": "ppippppippipp", "chiron_verify_workspace_bytes": "iii", "chiron_op_verify_drafts": "piiippppp",
        "chiron_op_linear4": "ppipipp", "chiron_linear4_workspace_bytes": "pi"}
_TYPES = {"p": C.c_void_p, "i": C.c_int32, "l": C.c_int64}


def load():
    """Load the built library; raises if it is missing (there is no other implementation)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libchiron.so is not built: run `python -m paper_2501_08090_amd.build` "
                              "(or __graft_entry__.build()); there is no fallback path")
        lib = C.CDLL(LIB_PATH)
        lib.chiron_last_error.restype = C.c_char_p
        lib.chiron_kv_block_bytes.restype = C.c_int64
        lib.chiron_kv_index_bytes.restype = C.c_int64
        lib.chiron_verify_workspace_bytes.restype = C.c_int64
        lib.chiron_linear4_workspace_bytes.restype = C.c_int64
        for name, types in _HOT.items():
            getattr(lib, name).argtypes = [_TYPES[t] for t in types]
        _lib = lib
    return _lib


def _check(rc):
    if rc != 0:
        raise ChironError(rc, load().chiron_last_error().decode())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t, dtype=None):
    if t is None:
        return C.c_void_p(0)
    if not t.is_cuda:
        raise TypeError("expected a GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError("expected %s, got %s" % (dtype, t.dtype))
    if not t.is_contiguous():
        raise TypeError("expected a contiguous tensor")
    return C.c_void_p(t.data_ptr())


_whole = index  # where an argument has the name
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _address(t, dtype=None):
    """_ptr for the entry points of _HOT: the number itself"""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous() or (dtype is not None and t.dtype != dtype):
        return _ptr(t, dtype)  # raises
    return t.data_ptr()


def _stream_number():
    """_stream for the entry points of _HOT"""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch._C._cuda_getDevice())


_ROW_TYPES = {torch.float32: CHIRON_F32, torch.bfloat16: CHIRON_BF16}


def _rows_of(t, rows, heads, d, dtype):
    """address and row stride of t [rows, heads, d], heads and dims contiguous"""
    if not t.is_cuda:
        raise TypeError("expected a GPU tensor")
    if t.dtype != dtype:
        raise TypeError("expected %s, got %s" % (dtype, t.dtype))
    if t.shape != (rows, heads, d):
        raise ValueError("expected [%d, %d, %d], got %s" % (rows, heads, d, tuple(t.shape)))
    s0, s1, s2 = t.stride()
    if rows < 2:
        s0 = heads * d
    if s2 != 1 or (s1 != d and heads > 1) or s0 < heads * d:
        raise TypeError("heads and dims of a row must be contiguous")
    return t.data_ptr(), s0


def make_config(m, max_batch, max_blocks_per_seq):
    return ModelConfig(m["n_layers"], m["hidden"], m["n_q_heads"], m["n_kv_heads"], m["head_dim"], m["ffn"], m["vocab"],
                       m["rope_base"], m["rms_eps"], CHIRON_BF16, int(max_batch), int(max_blocks_per_seq))


class Model:
    def __init__(self, m, max_batch, max_blocks_per_seq):
        self.cfg = make_config(m, max_batch, max_blocks_per_seq)
        self.shape = dict(m)
        self._h = C.c_void_p()
        _check(load().chiron_model_create(C.byref(self.cfg), C.byref(self._h)))

    def load_layer(self, layer, **w):
        lw = LayerWeights(*[_ptr(w[n], torch.bfloat16) for n, _ in LayerWeights._fields_])
        _check(load().chiron_model_load_layer(self._h, C.c_int32(layer), C.byref(lw), _stream()))

    def load_head(self, embed, final_norm, lm_head):
        _check(load().chiron_model_load_head(self._h, _ptr(embed, torch.bfloat16), _ptr(final_norm, torch.bfloat16),
                                             _ptr(lm_head, torch.bfloat16), _stream()))

    def load_weights(self, w):
        """w: dict as produced by inputs.make_weights (tensors on the GPU)."""
        for l in range(self.cfg.n_layers):
            self.load_layer(l, **{n: w[n][l] for n, _ in LayerWeights._fields_})
        self.load_head(w["embed"], w["final_norm"], w["lm_head"])

    def kv_block_bytes(self, block_size=16):
        return int(load().chiron_kv_block_bytes(self._h, C.c_int32(block_size)))

    def close(self):
        if self._h:
            torch.cuda.synchronize()
            load().chiron_model_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVPool:
    """Pool descriptor over a torch-allocated byte buffer (the caller owns the memory)."""

    def __init__(self, model, num_blocks=None, memory=None, block_size=16):
        self.model = model
        if memory is None:
            memory = torch.empty(int(num_blocks) * model.kv_block_bytes(block_size), dtype=torch.uint8, device="cuda")
        self.memory = memory
        self._h = C.c_void_p()
        nb = C.c_int32()
        _check(load().chiron_kv_pool_create(model._h, _ptr(memory), C.c_uint64(memory.numel() * memory.element_size()),
                                            C.c_int32(block_size), C.byref(self._h), C.byref(nb)))
        self.num_blocks = nb.value
        self.block_size = block_size
        self._views = {}  # layer -> torch views of the memory

    def append(self, layer, k, v, block_table, seq_idx, pos):
        n = seq_idx.numel()
        _check(load().chiron_append_kv(self._h, index(layer), _address(k, torch.bfloat16), _address(v, torch.bfloat16),
                                       _address(block_table, torch.int32), block_table.shape[1],
                                       _address(seq_idx, torch.int32), _address(pos, torch.int32), n, _stream_number()))

    def gather(self, layer, block_table_row, length):
        cfg = self.model.cfg
        k = torch.empty((length, cfg.n_kv_heads, cfg.head_dim), dtype=torch.bfloat16, device="cuda")
        v = torch.empty_like(k)
        _check(load().chiron_gather_kv(self._h, index(layer), _address(block_table_row, torch.int32), index(length), k.data_ptr(), v.data_ptr(),
                                       _stream_number()))
        return k, v

    def append_rope(self, layer, k, v, cos, sin, block_table, row_starts, seq_lens, q=None, index=None, q_out=None):
        """Rotate q and k by the rows' angles and write k and v behind the tokens already cached.

        k, v [rows, n_kv_heads, head_dim], q [rows, n_q_heads, head_dim]: fp32 or bf16 alike, rows of any stride (slices of a fused
        projection's rows, for one); cos, sin fp32 [rows, head_dim/2] (rope_table); request i brings the rows row_starts[i] ..
        row_starts[i+1]-1 at the positions from seq_lens[i] on.  index: a KVIndex to bring up to date.  Returns the rotated q, fp32."""
        cfg = self.model.cfg
        rows, batch, d, dtype = k.shape[0], seq_lens.numel(), cfg.head_dim, k.dtype
        if dtype not in _ROW_TYPES:
            raise TypeError("expected torch.float32 or torch.bfloat16, got %s" % dtype)
        width = block_table.shape[1] if block_table.dim() == 2 else -1
        if width < 0 or block_table.shape[0] < batch or row_starts.numel() != batch + 1:
            raise ValueError("%d requests need %d row starts and as many rows of the block table, got %d and %s" % (
                batch, batch + 1, row_starts.numel(), tuple(block_table.shape)))
        if cos.numel() != rows * (d // 2) or sin.numel() != cos.numel():
            raise ValueError("cos and sin must be [%d, %d], got %s and %s" % (rows, d // 2, tuple(cos.shape), tuple(sin.shape)))
        kp, ks = _rows_of(k, rows, cfg.n_kv_heads, d, dtype)
        vp, vs = _rows_of(v, rows, cfg.n_kv_heads, d, dtype)
        qp = qs = heads = out = 0
        if q is not None:
            heads = q.shape[1]
            qp, qs = _rows_of(q, rows, heads, d, dtype)
            if q_out is None:
                q_out = q.new_empty((rows, heads, d)) if dtype is torch.float32 else torch.empty((rows, heads, d), dtype=torch.float32, device=q.device)
            elif q_out.shape != q.shape:
                raise ValueError("q_out must have q's shape %s, got %s" % (tuple(q.shape), tuple(q_out.shape)))
            out = _address(q_out, torch.float32)
        r = NewRows(qp, kp, vp, qs, ks, vs, _ROW_TYPES[dtype], heads, _address(cos, torch.float32), _address(sin, torch.float32), out)
        _check(load().chiron_append_kv_rope(self._h, index._h if index is not None else None, _whole(layer), C.addressof(r),
                                            _address(block_table, torch.int32), width, _address(row_starts, torch.int32),
                                            _address(seq_lens, torch.int32), batch, rows, _stream_number()))
        return q_out

    def layer_views(self, layer):
        """The pool's memory of one layer as torch views without a copy: K [page, token, head, d/8, 8] and V [page, 4, 4 (token),
        head, d/32, 2, 16]; reshape either to [page, 16, head, d] for a copy in logical order."""
        layer = index(layer)
        if layer in self._views:
            return self._views[layer]
        cfg, nb = self.model.cfg, self.num_blocks
        n, d = cfg.n_kv_heads, cfg.head_dim
        if not 0 <= layer < cfg.n_layers:
            raise IndexError("layer %d out of range" % layer)
        size = nb * n * 2 * 16 * d
        t = self.memory.view(torch.uint8).view(-1)[layer * size * 2:(layer + 1) * size * 2].view(torch.bfloat16).view(nb, n, 2, 16 * d)
        k = t[:, :, 0].unflatten(2, (d // 8, 16, 8)).permute(0, 3, 1, 2, 4)
        v = t[:, :, 1].unflatten(2, (d // 32, 4, 16, 2, 4)).permute(0, 3, 6, 1, 2, 5, 4)
        self._views[layer] = (k, v)
        return k, v

    def swap_out(self, block_table_row, n_pages, image):
        """image: uint8 tensor of n_pages*block_bytes, on the GPU or in pinned host memory"""
        _check(load().chiron_kv_swap_out(self._h, _address(block_table_row, torch.int32), int(n_pages), image.data_ptr(),
                                         _stream_number()))

    def swap_in(self, block_table_row, n_pages, image):
        _check(load().chiron_kv_swap_in(self._h, _address(block_table_row, torch.int32), int(n_pages), image.data_ptr(),
                                        _stream_number()))

    def close(self):
        if self._h:
            load().chiron_kv_pool_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVIndex:
    """The page index of a pool, over a torch-allocated byte buffer (the caller owns the memory): per layer, page and KV head the
    bounds of the page's keys, which op_select_pages scores pages by."""

    def __init__(self, pool, memory=None):
        self.pool = pool
        need = int(load().chiron_kv_index_bytes(pool._h))
        if memory is None:
            memory = torch.zeros(need, dtype=torch.uint8, device="cuda")
        self.memory = memory
        self._h = C.c_void_p()
        _check(load().chiron_kv_index_create(pool._h, _ptr(memory), C.c_uint64(memory.numel() * memory.element_size()), C.byref(self._h)))

    def update(self, block_table, first, end, max_new, layer=0, n_layers=None):
        """Recompute the records of the pages that hold the positions first[i] .. end[i]-1 of each request (max_new at most), of
        all layers unless told otherwise."""
        cfg = self.pool.model.cfg
        batch = first.numel()
        if end.numel() != batch or block_table.dim() != 2 or block_table.shape[0] < batch:
            raise ValueError("first, end and the block table must have a row for each request")
        _check(load().chiron_kv_index_update(self._h, self.pool._h, index(layer), cfg.n_layers - layer if n_layers is None else index(n_layers),
                                             _address(block_table, torch.int32), block_table.shape[1], _address(first, torch.int32),
                                             _address(end, torch.int32), batch, index(max_new), _stream_number()))

    def layer_views(self, layer):
        """One layer's records as torch views without a copy: codes int8 [page, head, 2 (from above, from below), head_dim] and
        exponents int8 [page, head]; a bound is code * 2^exponent."""
        cfg, nb = self.pool.model.cfg, self.pool.num_blocks
        n, d, layer = cfg.n_kv_heads, cfg.head_dim, index(layer)
        if not 0 <= layer < cfg.n_layers:
            raise IndexError("layer %d out of range" % layer)
        size = (nb * n * (2 * d + 1) + 255) // 256 * 256
        t = self.memory.view(torch.uint8).view(-1)[layer * size:(layer + 1) * size].view(torch.int8)
        return t[:nb * n * 2 * d].view(nb, n, 2, d), t[nb * n * 2 * d:nb * n * (2 * d + 1)].view(nb, n)

    def close(self):
        if self._h:
            load().chiron_kv_index_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _check_table(model, block_table, batch):
    """The library indexes the block table with the model's max_blocks_per_seq as row stride."""
    if block_table.dim() != 2 or block_table.shape[1] != model.cfg.max_blocks_per_seq:
        raise ValueError("block_table must be [rows, %d] (the model's max_blocks_per_seq), got %s" % (
            model.cfg.max_blocks_per_seq, tuple(block_table.shape)))
    if block_table.shape[0] < batch:
        raise ValueError("block_table has %d rows for a batch of %d" % (block_table.shape[0], batch))


def decode_step(model, pool, block_table, seq_lens, tokens, logits=None, batch=None):
    B = seq_lens.numel() if batch is None else int(batch)
    _check_table(model, block_table, B)
    if logits is None:
        logits = torch.empty((B, model.cfg.vocab), dtype=torch.float32, device="cuda")
    _check(load().chiron_decode_step(model._h, pool._h, _address(block_table, torch.int32), _address(seq_lens, torch.int32),
                                     _address(tokens, torch.int32), B, _address(logits, torch.float32), _stream_number()))
    return logits


def decode_step_multi(model, pool, block_table, seq_lens, tokens, logits=None):
    """tokens [batch, q_len] int32 -> logits [batch, q_len, vocab]"""
    B, T = tokens.shape
    _check_table(model, block_table, B)
    if logits is None:
        logits = torch.empty((B, T, model.cfg.vocab), dtype=torch.float32, device="cuda")
    _check(load().chiron_decode_step_multi(model._h, pool._h, _address(block_table, torch.int32), _address(seq_lens, torch.int32),
                                           _address(tokens, torch.int32), B, T, _address(logits, torch.float32), _stream_number()))
    return logits


def validate_step_inputs(model, pool, block_table, seq_lens, tokens, batch=None):
    """tokens [batch] or, for the multi-token step, [batch, q_len]"""
    B = seq_lens.numel() if batch is None else int(batch)
    _check_table(model, block_table, B)
    if tokens.dim() == 2:
        _check(load().chiron_validate_step_inputs_multi(model._h, pool._h, _ptr(block_table, torch.int32), _ptr(seq_lens, torch.int32),
                                                        _ptr(tokens, torch.int32), C.c_int32(B), C.c_int32(tokens.shape[1]), _stream()))
        return
    _check(load().chiron_validate_step_inputs(model._h, pool._h, _ptr(block_table, torch.int32), _ptr(seq_lens, torch.int32),
                                              _ptr(tokens, torch.int32), C.c_int32(B), _stream()))


def check_step_inputs_host(cfg, num_blocks, block_table, seq_lens, tokens, block_size=16):
    """Host-only check of index arrays (numpy int32); tokens [batch] or [batch, q_len]."""
    import numpy as np
    bt = np.ascontiguousarray(block_table, np.int32)
    sl = np.ascontiguousarray(seq_lens, np.int32)
    tk = np.ascontiguousarray(tokens, np.int32)
    p = lambda a: a.ctypes.data_as(C.c_void_p)
    if tk.ndim == 2:
        return int(load().chiron_check_step_inputs_host_multi(C.byref(cfg), C.c_int32(num_blocks), C.c_int32(block_size), p(bt),
                                                              p(sl), p(tk), C.c_int32(sl.size), C.c_int32(tk.shape[1])))
    return int(load().chiron_check_step_inputs_host(C.byref(cfg), C.c_int32(num_blocks), C.c_int32(block_size), p(bt), p(sl),
                                                    p(tk), C.c_int32(sl.size)))


def last_error():
    return load().chiron_last_error().decode()


def step_latency_profile(model, pool, block_table, seq_lens, tokens, batch_sizes, warmup=2, iters=5, logits=None):
    n = len(batch_sizes)
    _check_table(model, block_table, max(batch_sizes))
    if logits is None:
        logits = torch.empty((max(batch_sizes), model.cfg.vocab), dtype=torch.float32, device="cuda")
    bs = (C.c_int32 * n)(*batch_sizes)
    out = (ProfilePoint * n)()
    _check(load().chiron_step_latency_profile(model._h, pool._h, _ptr(block_table, torch.int32), _ptr(seq_lens, torch.int32),
                                              _ptr(tokens, torch.int32), bs, C.c_int32(n), C.c_int32(warmup), C.c_int32(iters),
                                              _ptr(logits, torch.float32), _stream(), out))
    return [dict(batch=p.batch, lat_ms_median=p.lat_ms_median, lat_ms_p99=p.lat_ms_p99, lat_ms_mean=p.lat_ms_mean,
                 tokens_per_s=p.tokens_per_s) for p in out]


def local_autoscale_step(itl, itl_slo, tput_prev, tput_curr, max_batch, batch_limit, alpha=0.5):
    """One update of the maximum batch size (host arithmetic).  -> (new max batch, local backpressure)"""
    mb = C.c_int32(int(max_batch))
    lb = C.c_double()
    _check(load().chiron_local_autoscale_step(C.c_double(itl), C.c_double(itl_slo), C.c_double(tput_prev), C.c_double(tput_curr),
                                              C.c_double(alpha), C.c_int32(int(batch_limit)), C.byref(mb), C.byref(lb)))
    return mb.value, lb.value


KERNEL_CLASSES = ("qkv", "o", "gateup", "down", "lmhead", "attn", "attn_merge", "rmsnorm", "rope_append", "other")


class KernelTime(C.Structure):
    _fields_ = [("ms", C.c_double), ("launches", C.c_int64)]


def kernel_timing_begin(model):
    _check(load().chiron_kernel_timing_begin(model._h))


def kernel_timing_end(model):
    """-> {class: (total_ms, launches)}"""
    out = (KernelTime * len(KERNEL_CLASSES))()
    _check(load().chiron_kernel_timing_end(model._h, _stream(), out))
    return {n: (out[i].ms, int(out[i].launches)) for i, n in enumerate(KERNEL_CLASSES)}


# ---- single kernels -------------------------------------------------------------------------------

def op_rmsnorm(h, gain, eps):
    out = torch.empty_like(h)
    _check(load().chiron_op_rmsnorm(_ptr(h, torch.float32), _ptr(gain, torch.bfloat16), C.c_int32(h.shape[0]),
                                    C.c_int32(h.shape[1]), C.c_float(eps), _ptr(out), _stream()))
    return out


class Linear:
    def __init__(self, w):
        self.N, self.K = w.shape
        self._h = C.c_void_p()
        _check(load().chiron_linear_create(_ptr(w, torch.bfloat16), C.c_int32(self.N), C.c_int32(self.K), _stream(),
                                           C.byref(self._h)))

    def __call__(self, x, y=None, accumulate=False):
        M = x.shape[0]
        if y is None:
            y = torch.empty((M, self.N), dtype=torch.float32, device="cuda")
        _check(load().chiron_op_linear(self._h, _address(x, torch.float32), M, _address(y, torch.float32), 1 if accumulate else 0,
                                       _stream_number()))
        return y

    def close(self):
        if self._h:
            torch.cuda.synchronize()
            load().chiron_linear_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GateUp(Linear):
    """The fused gate/up matrix of a feed-forward block (w_gate, w_up [F, K] bf16)."""

    def __init__(self, w_gate, w_up):
        self.F, self.K = w_gate.shape
        if tuple(w_up.shape) != (self.F, self.K):
            raise ValueError("w_gate and w_up differ in shape")
        self.N = 2 * self.F
        self._h = C.c_void_p()
        _check(load().chiron_linear_create_gate_up(_ptr(w_gate, torch.bfloat16), _ptr(w_up, torch.bfloat16), C.c_int32(self.F),
                                                   C.c_int32(self.K), _stream(), C.byref(self._h)))

    def __call__(self, x, *a, **k):
        raise TypeError("a fused gate/up matrix has no plain product: use swiglu() or ffn()")

    def swiglu(self, x):
        """silu(x Wg^T) * (x Wu^T), fp32 [M, F]"""
        M = x.shape[0]
        act = torch.empty((M, self.F), dtype=torch.float32, device="cuda")
        _check(load().chiron_op_gate_up_swiglu(self._h, _address(x, torch.float32), M, _address(act, torch.float32), _stream_number()))
        return act

    def ffn(self, down, x, y=None, accumulate=False):
        """y (+)= (silu(x Wg^T) * (x Wu^T)) Wd^T with down = Linear(Wd)"""
        M = x.shape[0]
        if y is None:
            y = torch.empty((M, down.N), dtype=torch.float32, device="cuda")
        _check(load().chiron_op_swiglu_ffn(self._h, down._h, _address(x, torch.float32), M, _address(y, torch.float32),
                                           1 if accumulate else 0, _stream_number()))
        return y


def set_tuning(key, value):
    _check(load().chiron_set_tuning(key.encode(), C.c_int32(int(value))))


def op_rope(x, pos, base):
    """x [rows, n_heads, d] fp32, rotated in place."""
    rows, nh, d = x.shape
    _check(load().chiron_op_rope(_ptr(x, torch.float32), C.c_int32(rows), C.c_int32(nh), C.c_int32(d), _ptr(pos, torch.int32),
                                 C.c_float(base), _stream()))
    return x


def op_rope_noalloc(x, pos, base):
    """op_rope through the entry point that allocates nothing (fixed table inside the library)."""
    rows, nh, d = x.shape
    _check(load().chiron_op_rope_noalloc(_ptr(x, torch.float32), C.c_int32(rows), C.c_int32(nh), C.c_int32(d),
                                         _ptr(pos, torch.int32), C.c_float(base), _stream()))
    return x


def op_paged_attention(model, pool, layer, q, block_table, ctx_lens):
    B = ctx_lens.numel()
    _check_table(model, block_table, B)
    out = torch.empty_like(q)
    _check(load().chiron_op_paged_attention(model._h, pool._h, index(layer), _address(q, torch.float32), _address(block_table, torch.int32),
                                            _address(ctx_lens, torch.int32), B, _address(out), _stream_number()))
    return out


# ---- drafting: block-sparse attention, verification, 4-bit products ---------------------------------------------------

def rope_table(pos, d, base):
    """cos and sin [rows, d/2] fp32 of pos[r] * base^(-2j/d), pos int32: one table for all layers of a step"""
    rows = pos.numel()
    cos = torch.empty((rows, d // 2), dtype=torch.float32, device=pos.device)
    sin = torch.empty_like(cos)
    _check(load().chiron_op_rope_table(_ptr(pos, torch.int32), C.c_int32(rows), C.c_int32(d), C.c_float(base), _ptr(cos), _ptr(sin), _stream()))
    return cos, sin


def _check_rows(model, q, block_table, ctx_lens, row_seq):
    rows = ctx_lens.numel()
    _check_table(model, block_table, rows if row_seq is None else 0)
    if q.numel() != rows * model.cfg.n_q_heads * model.cfg.head_dim:
        raise ValueError("q must hold %d rows of %d values, got %s" % (rows, model.cfg.n_q_heads * model.cfg.head_dim, tuple(q.shape)))
    if row_seq is not None and row_seq.numel() != rows:
        raise ValueError("row_seq must name a request for each of %d rows, got %d" % (rows, row_seq.numel()))
    return rows


def op_select_pages(model, pool, kv_index, layer, q, block_table, ctx_lens, top, n_first=1, n_last=1, row_seq=None):
    """The pages that each row of q (fp32, rotated) attends, chosen by the page index.  Row r is a token of request row_seq[r] (of
    request r without it) that sees ctx_lens[r] positions.  -> pages int32 [rows, n_kv_heads, top] ascending, then -1; counts int32 [rows]"""
    rows, top = _check_rows(model, q, block_table, ctx_lens, row_seq), index(top)
    pages, counts = ctx_lens.new_empty((rows, model.cfg.n_kv_heads, max(top, 0))), ctx_lens.new_empty(rows)
    _check(load().chiron_op_select_pages(model._h, pool._h, kv_index._h, index(layer), _address(q, torch.float32), _address(block_table, torch.int32),
                                         _address(row_seq, torch.int32), _address(ctx_lens, torch.int32), rows, top, index(n_first),
                                         index(n_last), _address(pages), _address(counts), _stream_number()))
    return pages, counts


def op_sparse_attention(model, pool, layer, q, block_table, ctx_lens, pages, counts=None, row_seq=None):
    """Attention of each row over the tokens of its listed pages (op_select_pages, or lists of the caller's own)"""
    rows = _check_rows(model, q, block_table, ctx_lens, row_seq)
    if pages.dim() != 3 or pages.shape[0] != rows or pages.shape[1] != model.cfg.n_kv_heads:
        raise ValueError("pages must be [%d, %d, top], got %s" % (rows, model.cfg.n_kv_heads, tuple(pages.shape)))
    if counts is not None and counts.numel() != rows:
        raise ValueError("counts must have %d entries, got %d" % (rows, counts.numel()))
    out = torch.empty_like(q)
    _check(load().chiron_op_sparse_attention(model._h, pool._h, index(layer), _address(q, torch.float32), _address(block_table, torch.int32),
                                             _address(row_seq, torch.int32), _address(ctx_lens, torch.int32), rows, _address(pages, torch.int32),
                                             _address(counts, torch.int32), pages.shape[2], _address(out), _stream_number()))
    return out


def _logit_rows(t, batch, rows, vocab):
    """address and row stride of t [batch, rows, vocab] fp32: rows of any stride, requests one behind the other"""
    if not t.is_cuda:
        raise TypeError("expected a GPU tensor")
    if t.dtype != torch.float32:
        raise TypeError("expected %s, got %s" % (torch.float32, t.dtype))
    if t.shape != (batch, rows, vocab):
        raise ValueError("expected logits [%d, %d, %d], got %s" % (batch, rows, vocab, tuple(t.shape)))
    stride = t.stride(1) if rows > 1 else t.stride(0) if batch > 1 else vocab
    if (vocab > 1 and t.stride(2) != 1) or (batch > 1 and rows > 0 and t.stride(0) != rows * stride):
        raise TypeError("logits must be contiguous but for their row stride")
    return t.data_ptr() or None, stride


_verify_work = {}  # (requests, drafts, vocabulary) -> 4-byte words of workspace


def verify_drafts(logits, tokens, uniforms, noise, draft_logits=None, draft_lens=None, temperature=None):
    """Accept or replace drafted tokens.  logits fp32 [batch, drafts+1, vocab] of the target, tokens int32 [batch, drafts], uniforms fp32
    [batch, drafts] in [0, 1), noise fp32 [batch, vocab] from the unit exponential distribution, draft_logits fp32 [batch, drafts,
    vocab] or None (drafts that were not sampled), draft_lens int32 [batch], temperature fp32 [batch] (0: greedy).  At most 127 drafts,
    and batch * (2 drafts + 1) at most 65535.
    -> tokens int32 [batch, drafts+1] (the accepted ones, the new one, then -1), accepted int32 [batch], prob fp32 [batch, drafts]"""
    batch, rows, vocab = logits.shape
    drafts = rows - 1
    if tokens.shape != (batch, drafts) or uniforms.shape != (batch, drafts) or noise.shape != (batch, vocab):
        raise ValueError("%d requests of %d drafts over %d tokens: got tokens %s, uniforms %s, noise %s" % (
            batch, drafts, vocab, tuple(tokens.shape), tuple(uniforms.shape), tuple(noise.shape)))
    for t in (draft_lens, temperature):
        if t is not None and t.numel() != batch:
            raise ValueError("draft_lens and temperature must have %d entries, got %d" % (batch, t.numel()))
    b = DraftBatch()
    b.logits, b.logits_stride = _logit_rows(logits, batch, rows, vocab)
    if draft_logits is not None and drafts > 0:
        b.draft_logits, b.draft_stride = _logit_rows(draft_logits, batch, drafts, vocab)
    b.tokens, b.draft_lens = _address(tokens, torch.int32), _address(draft_lens, torch.int32)
    b.uniforms, b.noise, b.temperature = _address(uniforms, torch.float32), _address(noise, torch.float32), _address(temperature, torch.float32)
    need = _verify_work.get((batch, drafts, vocab))
    if need is None:
        need = _verify_work[batch, drafts, vocab] = load().chiron_verify_workspace_bytes(batch, drafts, vocab) // 4
    work, out, accepted, prob = tokens.new_empty(need), tokens.new_empty((batch, rows)), tokens.new_empty(batch), torch.empty_like(uniforms)
    _check(load().chiron_op_verify_drafts(C.addressof(b), batch, drafts, vocab, out.data_ptr() or None, accepted.data_ptr() or None,
                                          prob.data_ptr() or None, work.data_ptr() or None, _stream_number()))
    return out, accepted, prob


class Linear4:
    """A matrix of 4-bit weights: W[n][k] = (w4[n][k] - zero[n][k // group]) * scale[n][k // group].  w4 uint8 [N, K/2] (even k in the
    low bits), scales bf16 [N, K/group], zeros uint8 [N, K/group], 0 .. 64, or None (8); group 32, 64 or 128."""

    def __init__(self, w4, scales, zeros=None):
        self.N, self.K = w4.shape[0], 2 * w4.shape[1]
        groups = scales.shape[1]
        if scales.shape[0] != self.N or groups < 1 or self.K % groups != 0 or (zeros is not None and zeros.shape != scales.shape):
            raise ValueError("w4 %s, scales %s and zeros %s do not fit" % (tuple(w4.shape), tuple(scales.shape), None if zeros is None else tuple(zeros.shape)))
        self.group = self.K // groups
        self._work = {}  # rows -> bytes of workspace
        self._h = C.c_void_p()
        _check(load().chiron_linear4_create(_ptr(w4, torch.uint8), _ptr(scales, torch.bfloat16), _ptr(zeros, torch.uint8), C.c_int32(self.N),
                                            C.c_int32(self.K), C.c_int32(self.group), _stream(), C.byref(self._h)))

    def __call__(self, x, y=None, accumulate=False):
        M = x.shape[0]
        if x.numel() != M * self.K:
            raise ValueError("x must be [rows, %d], got %s" % (self.K, tuple(x.shape)))
        if y is None:
            if accumulate:
                raise ValueError("accumulate needs y")
            y = x.new_empty((M, self.N))
        elif y.numel() != M * self.N:
            raise ValueError("y must be [%d, %d], got %s" % (M, self.N, tuple(y.shape)))
        need = self._work.get(M)
        if need is None:
            need = self._work[M] = load().chiron_linear4_workspace_bytes(self._h, M)
        work = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        _check(load().chiron_op_linear4(self._h, _address(x, torch.float32), M, _address(y, torch.float32), 1 if accumulate else 0,
                                        _address(work), _stream_number()))
        return y

    def close(self):
        if self._h:
            torch.cuda.synchronize()
            load().chiron_linear4_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
