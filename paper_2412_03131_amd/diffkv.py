"""Thin ctypes binding of libdiffkv.so (the C ABI declared in include/diffkv.h).

Argument marshalling only: every step of the hot path runs in the HIP
kernels of the library.  PyTorch provides device memory and the stream: the
current one, or the one that a call is given.  Buffers that a call is not given
come from its stream; a result that another stream uses is ordered by the
program, as torch's own are (wait_stream, record_stream).
Loading fails loudly when the library has not been built.
"""
import contextlib
import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdiffkv.so")

OK, E_INVAL, E_UNSUPPORTED, E_WORKSPACE, E_LAUNCH, E_SCRATCH = 0, 1, 2, 3, 4, 5
ST_OUT_OF_PAGES, ST_TABLE_OVERFLOW, ST_BAD_INPUT = 1, 2, 4
OP_APPEND, OP_ATTENTION, OP_COMPACT, OP_ALLOC, OP_GENERATION, OP_PROMPT_SIGNIFICANCE = 0, 1, 2, 3, 4, 5
OP_CHUNK_ATTENTION, OP_CHUNK_SIGNIFICANCE, OP_BLOCK_ATTENTION = 6, 7, 8
HIGH, LOW = 0, 1
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BY_PARTS = 0, 1, 2, 3
BLOCK_TOKENS = 32
BLOCK_E4M3, BLOCK_INT8 = 0, 1

_lib = None


class DiffKVError(RuntimeError):
    def __init__(self, code, what):
        super().__init__("%s: %s (status %d)" % (what, status_str(code), code))
        self.code = code


class Layout(C.Structure):
    _fields_ = [
        ("head_dim", C.c_int32), ("group", C.c_int32),
        ("k_bits", C.c_int32 * 2), ("v_bits", C.c_int32 * 2),
        ("tokens_per_page", C.c_int32 * 2),
        ("max_seq_len", C.c_int32), ("p_max", C.c_int32),
        ("page_bytes", C.c_int64),
        ("off_kcode", C.c_int32 * 2), ("off_kmeta", C.c_int32 * 2),
        ("off_vcode", C.c_int32 * 2), ("off_vmeta", C.c_int32 * 2),
        ("off_score", C.c_int32 * 2), ("off_pos", C.c_int32 * 2),
        ("used_bytes", C.c_int32 * 2),
    ]


class CacheStruct(C.Structure):
    _fields_ = [
        ("pool", C.c_void_p), ("num_pages", C.c_int64),
        ("page_table", C.c_void_p), ("pages", C.c_void_p), ("len", C.c_void_p),
        ("seq_len", C.c_void_p), ("ring", C.c_void_p), ("ring_ptr", C.c_void_p),
        ("status", C.c_void_p), ("num_seqs", C.c_int32), ("num_kv_heads", C.c_int32),
    ]


class ScoreForm(C.Structure):
    _fields_ = [("cap", C.c_float), ("window", C.c_int32), ("slopes", C.c_void_p)]


class BlockCacheStruct(C.Structure):
    _fields_ = [
        ("pool", C.c_void_p), ("scale", C.c_void_p), ("num_blocks", C.c_int64), ("table", C.c_void_p),
        ("tail", C.c_void_p), ("seq_len", C.c_void_p), ("status", C.c_void_p), ("num_seqs", C.c_int32),
        ("num_kv_heads", C.c_int32), ("format", C.c_int32),
    ]


EXPORTS = ("diffkv_layout_init", "diffkv_workspace_size", "diffkv_quantize_append",
           "diffkv_decode_attention", "diffkv_decode_attention_noalloc", "diffkv_update_significance",
           "diffkv_prompt_significance", "diffkv_rotate", "diffkv_rope_frequencies", "diffkv_chunk_attention",
           "diffkv_chunk_significance", "diffkv_norm_rotate", "diffkv_block_append", "diffkv_block_read",
           "diffkv_block_attention", "diffkv_compact_free_list", "diffkv_alloc_pages",
           "diffkv_generation_step", "diffkv_status_str")


def lib():
    """Load libdiffkv.so (raises if it is missing: there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libdiffkv.so is not built (%s); run __graft_entry__.build()" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        PL = C.POINTER(Layout)
        PC = C.POINTER(CacheStruct)
        L.diffkv_layout_init.argtypes = [PL, i32, i32, vp, vp, vp, i32]
        L.diffkv_workspace_size.argtypes = [i32, PL, i32, i32, i32, i64, i32, C.POINTER(sz)]
        L.diffkv_quantize_append.argtypes = [PL, PC, i64, i32, vp, vp, vp, vp, vp, f32, f32, i32,
                                             vp, sz, vp]
        L.diffkv_decode_attention.argtypes = [PL, PC, i32, vp, f32, vp, vp, i32, vp, sz, vp]
        L.diffkv_decode_attention_noalloc.argtypes = [PL, PC, i32, vp, f32, vp, vp, i32, vp]
        L.diffkv_update_significance.argtypes = [PL, PC, i32, vp, f32, vp, vp]
        L.diffkv_prompt_significance.argtypes = [PL, i32, i64, i32, vp, i32, i32, vp, vp, f32, vp, vp,
                                                 vp, sz, vp]
        PF = C.POINTER(ScoreForm)
        L.diffkv_rotate.argtypes = [PL, i64, vp, vp, i32, i32, f32, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64, vp]
        L.diffkv_rope_frequencies.argtypes = [i32, C.c_double, i32, C.c_double, i32, C.c_double, C.c_double, vp, vp]
        L.diffkv_chunk_attention.argtypes = [PL, PC, i64, i32, vp, i32, vp, i64, vp, i64, vp, i64, f32, PF, vp, vp,
                                             vp, sz, vp]
        L.diffkv_chunk_significance.argtypes = [PL, PC, i64, i32, vp, i32, vp, i64, vp, i64, f32, PF, vp, vp,
                                                vp, sz, vp]
        PB = C.POINTER(BlockCacheStruct)
        L.diffkv_norm_rotate.argtypes = [PL, i64, vp, vp, i32, i32, f32, f32, i32, vp, i64, vp, vp, i64,
                                         i32, vp, i64, vp, vp, i64, vp]
        L.diffkv_block_append.argtypes = [PL, PB, i64, i32, vp, vp, i64, vp, i64, vp]
        L.diffkv_block_read.argtypes = [PL, PB, i64, i32, vp, vp, vp, i64, vp, i64, vp]
        L.diffkv_block_attention.argtypes = [PL, PB, i64, i32, vp, i32, vp, i64, vp, i64, vp, i64, f32, PF, i32, vp, vp,
                                             vp, sz, vp]
        L.diffkv_compact_free_list.argtypes = [PL, PC, i32, vp, vp, sz, vp]
        L.diffkv_alloc_pages.argtypes = [PL, PC, i32, vp, vp, sz, vp]
        L.diffkv_generation_step.argtypes = [PL, PC, f32, f32, i32, vp, sz, vp]
        L.diffkv_status_str.argtypes = [i32]
        L.diffkv_status_str.restype = C.c_char_p
        for n in EXPORTS[:-1]:
            getattr(L, n).restype = i32
        _lib = L
    return _lib


def status_str(code):
    return lib().diffkv_status_str(code).decode()


def _check(code, what):
    if code != OK:
        raise DiffKVError(code, what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:  # the current device's current stream, as an address
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def layout(head_dim=128, group=32, k_bits=(8, 4), v_bits=(4, 2), tokens_per_page=(16, 32),
           max_seq_len=4096):
    L = Layout()
    kb = (C.c_int32 * 2)(*k_bits)
    vb = (C.c_int32 * 2)(*v_bits)
    tp = (C.c_int32 * 2)(*tokens_per_page)
    _check(lib().diffkv_layout_init(C.byref(L), head_dim, group, kb, vb, tp, max_seq_len),
           "diffkv_layout_init")
    return L


def workspace_size(op, L, num_seqs, num_q_heads=0, num_kv_heads=1, total_new=0, num_splits=0):
    n = C.c_size_t(0)
    _check(lib().diffkv_workspace_size(op, C.byref(L), num_seqs, num_q_heads, num_kv_heads,
                                       total_new, num_splits, C.byref(n)), "diffkv_workspace_size")
    return n.value


# The calls below cost the host what a short kernel costs the device, so what they
# marshal is kept to the call's own arguments: the cache's addresses packed into
# the structure at once, the stream's address, plain integers, and no size query for
# a workspace that the caller brings (the library checks its size).
_CACHE = struct.Struct("PqPPPPPPPii")
assert _CACHE.size == C.sizeof(CacheStruct)


def _cache_struct(c):
    return CacheStruct.from_buffer_copy(_CACHE.pack(
        c.pool.data_ptr(), c.num_pages, c.page_table.data_ptr(), c.pages.data_ptr(), c.len.data_ptr(),
        c.seq_len.data_ptr(), c.ring.data_ptr(), c.ring_ptr.data_ptr(), c.status.data_ptr(), c.num_seqs,
        c.num_kv_heads))


_HERE = contextlib.nullcontext()


def _on(stream):
    """What a call does before its launch (lengths read, buffers taken) is done on the stream that it runs on."""
    if stream is None or (stream.cuda_stream == _stream(None) and stream.device.index == torch._C._cuda_getDevice()):
        return _HERE
    return torch.cuda.stream(stream)


def _new(stream, shape, dtype, device):
    """A buffer that a call is not given, taken from its stream: the bytes of one taken from another may be in use there
    as the call's kernels start, or that stream's next buffer before they end."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _on(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _longest(lens, stream):
    """Read with a synchronization of the call's stream: where its kernels read the lengths, they are written by then."""
    with _on(stream):
        return int(lens.max().item()) if lens.shape[0] else 0


def _new_ws(nbytes, device, stream):
    return _new(stream, max(nbytes, 256), torch.uint8, device)


def _check_ws(code, what, *sizes):
    """As _check; a workspace that is too small is a ValueError that says what is needed."""
    if code == E_WORKSPACE:
        raise ValueError("workspace too small: need %d bytes" % workspace_size(*sizes))
    if code != OK:
        raise DiffKVError(code, what)


class Cache:
    """Device tensors of one cache (diffkv_cache); the library owns none of them."""

    def __init__(self, L, num_pages, num_seqs, num_kv_heads, device="cuda", ring=None,
                 with_pool=True):
        self.L = L
        self.num_pages = int(num_pages)
        self.num_seqs = int(num_seqs)
        self.num_kv_heads = int(num_kv_heads)
        T = self.num_seqs * self.num_kv_heads
        dev = torch.device(device)
        self.pool = torch.zeros((self.num_pages if with_pool else 1, L.page_bytes),
                                dtype=torch.uint8, device=dev)
        self.page_table = torch.full((T, L.p_max), -1, dtype=torch.int32, device=dev)
        self.pages = torch.zeros((T, 2), dtype=torch.int32, device=dev)
        self.len = torch.zeros((T, 2), dtype=torch.int32, device=dev)
        self.seq_len = torch.zeros(self.num_seqs, dtype=torch.int32, device=dev)
        if ring is None:
            self.ring = torch.arange(self.num_pages, dtype=torch.int32, device=dev)
        else:
            self.ring = torch.as_tensor(ring, dtype=torch.int32).to(dev).contiguous()
        self.ring_ptr = torch.tensor([0, self.num_pages], dtype=torch.int64, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)

    @property
    def num_tables(self):
        return self.num_seqs * self.num_kv_heads

    def view(self, seq_lo, seq_hi):
        """Cache over sequences [seq_lo, seq_hi) sharing this cache's pool, ring, pointers
        and status (e.g. one layer of a cache whose "sequences" are layer-major)."""
        v = Cache.__new__(Cache)
        v.L = self.L
        v.num_pages = self.num_pages
        v.num_seqs = seq_hi - seq_lo
        v.num_kv_heads = self.num_kv_heads
        H = self.num_kv_heads
        v.pool, v.ring, v.ring_ptr, v.status = self.pool, self.ring, self.ring_ptr, self.status
        v.page_table = self.page_table[seq_lo * H:seq_hi * H]
        v.pages = self.pages[seq_lo * H:seq_hi * H]
        v.len = self.len[seq_lo * H:seq_hi * H]
        v.seq_len = self.seq_len[seq_lo:seq_hi]
        return v

    def struct(self):
        return CacheStruct(self.pool.data_ptr(), self.num_pages, self.page_table.data_ptr(),
                           self.pages.data_ptr(), self.len.data_ptr(), self.seq_len.data_ptr(),
                           self.ring.data_ptr(), self.ring_ptr.data_ptr(), self.status.data_ptr(),
                           self.num_seqs, self.num_kv_heads)


def _bits16(t):
    return t if t.dtype in (torch.int16, torch.float16, torch.bfloat16) else t.view(torch.int16)


def quantize_append(cache, new_len, k, v, score, quota=None, alpha_h=0.0, alpha_l=0.0,
                    window=0, total_new=None, max_new=None, ws=None, stream=None):
    """new_len int32 [B] (device); k, v fp16 [total_new, Hkv, D]; score fp32 [total_new, Hkv];
    quota int32 [B, Hkv, 2] or None (threshold form).  total_new / max_new are host sizes
    (read from new_len with a device sync when omitted)."""
    L = cache.L
    if total_new is None or max_new is None:
        with _on(stream):
            nl = new_len.cpu()
        total_new = int(nl.sum()) if total_new is None else total_new
        max_new = int(nl.max()) if max_new is None else max_new
    sizes = (OP_APPEND, L, cache.num_seqs, 0, cache.num_kv_heads, total_new)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), cache.pool.device, stream)
    _check_ws(lib().diffkv_quantize_append(
        C.byref(L), _cache_struct(cache), int(total_new), int(max_new), _ptr(new_len), _ptr(_bits16(k)),
        _ptr(_bits16(v)), _ptr(score), _ptr(quota), float(alpha_h), float(alpha_l), int(window),
        ws.data_ptr(), ws.nbytes, _stream(stream)), "diffkv_quantize_append", *sizes)
    return ws


def decode_attention(cache, q, sm_scale, out=None, lse=None, num_splits=0, ws=None, stream=None,
                     want_lse=True):
    """q fp16 [B, Hq, D] (device) -> out fp32 [B, Hq, D], lse fp32 [B, Hq]."""
    L = cache.L
    B, Hq, D = q.shape
    if out is None:
        out = _new(stream, (B, Hq, D), torch.float32, q.device)
    if lse is None and want_lse:
        lse = _new(stream, (B, Hq), torch.float32, q.device)
    sizes = (OP_ATTENTION, L, cache.num_seqs, Hq, cache.num_kv_heads, 0, num_splits)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), q.device, stream)
    _check_ws(lib().diffkv_decode_attention(
        C.byref(L), _cache_struct(cache), Hq, _ptr(_bits16(q)), float(sm_scale), _ptr(out), _ptr(lse),
        int(num_splits), ws.data_ptr(), ws.nbytes, _stream(stream)), "diffkv_decode_attention", *sizes)
    return out, lse


def decode_attention_noalloc(cache, q, sm_scale, out, lse=None, num_splits=0, stream=None):
    """diffkv_decode_attention_noalloc: like decode_attention, outputs given by the
    caller, no workspace (the library's fixed per-device scratch)."""
    _check(lib().diffkv_decode_attention_noalloc(
        C.byref(cache.L), _cache_struct(cache), q.shape[1], _ptr(_bits16(q)), float(sm_scale), _ptr(out),
        _ptr(lse), int(num_splits), _stream(stream)), "diffkv_decode_attention_noalloc")
    return out, lse


def update_significance(cache, q, sm_scale, lse, stream=None):
    """diffkv_update_significance: every kept token's score becomes the running mean of
    its attention probability (max over the KV head's query heads); lse from
    decode_attention with the same q."""
    _check(lib().diffkv_update_significance(C.byref(cache.L), _cache_struct(cache), q.shape[1], _ptr(_bits16(q)),
                                            float(sm_scale), _ptr(lse), _stream(stream)),
           "diffkv_update_significance")


def prompt_significance(L, new_len, q, k, sm_scale, lse=None, score=None, max_new=None, ws=None,
                        stream=None):
    """diffkv_prompt_significance: q fp16 [rows, Hq, D], k fp16 [rows, Hkv, D] (device, rows
    concatenated per sequence), new_len int32 [B] (device); returns score fp32 [rows, Hkv].
    lse (fp32 [rows, Hq], natural log) skips the row pass when given."""
    rows, Hq, Hkv = q.shape[0], q.shape[1], k.shape[1]
    B = new_len.shape[0]
    if max_new is None:
        max_new = _longest(new_len, stream)
    if score is None:
        score = _new(stream, (rows, Hkv), torch.float32, q.device)
    sizes = (OP_PROMPT_SIGNIFICANCE, L, B, Hq, Hkv, rows)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), q.device, stream)
    _check_ws(lib().diffkv_prompt_significance(C.byref(L), B, rows, int(max_new), _ptr(new_len), Hq, Hkv,
                                               _ptr(_bits16(q)), _ptr(_bits16(k)), float(sm_scale), _ptr(lse),
                                               _ptr(score), ws.data_ptr(), ws.nbytes, _stream(stream)),
              "diffkv_prompt_significance", *sizes)
    return score


def _rows(t, what, head_dim):
    """Address and row stride of [rows, heads, D] rows whose heads lie side by side (a slice of a
    fused projection may be given)."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or t.dtype != torch.float16 or shape[2] != head_dim or stride[2] != 1 or (
            stride[1] != head_dim and shape[1] > 1):
        raise ValueError("%s: fp16 [rows, heads, %d] with packed heads expected" % (what, head_dim))
    return t.data_ptr(), stride[0]


def _on_one_gpu(what, *tensors):
    """All on the same GPU (None aside): an address of the host's would fault the device."""
    at = tensors[0].get_device()
    for t in tensors:
        if t is not None and (at < 0 or t.get_device() != at):
            raise ValueError("%s: tensors on one GPU expected" % what)


def _stream_at(what, stream, t):
    """A stream's address; it has to be one of the GPU that t is on (a kernel runs where its stream is).  Asked for
    before a call allocates or reads lengths, which it does there."""
    if t.get_device() < 0:
        raise ValueError("%s: tensors on one GPU expected" % what)
    if (torch._C._cuda_getDevice() if stream is None else stream.device.index) != t.get_device():
        raise ValueError("%s: a stream of the tensors' GPU expected (None: the current GPU's)" % what)
    return _stream(stream)


def _form(cap, window, slopes):
    if cap == 0.0 and window == 0 and slopes is None:
        return None
    return C.byref(ScoreForm(float(cap), int(window), _ptr(slopes)))


def rope_frequencies(rot_dim, base=10000.0, scaling=ROPE_PLAIN, factor=1.0, trained_len=0, slow=1.0, fast=32.0):
    """diffkv_rope_frequencies: (fp32 [rot_dim / 2] on the host, the scale of cosines and sines).  rotate takes
    them on the device."""
    freq = torch.empty(max(rot_dim // 2, 1), dtype=torch.float32)
    scale = C.c_float(0.0)
    _check(lib().diffkv_rope_frequencies(int(rot_dim), float(base), int(scaling), float(factor), int(trained_len),
                                         float(slow), float(fast), freq.data_ptr(), C.addressof(scale)),
           "diffkv_rope_frequencies")
    return freq, scale.value


def _rotate_args(what, L, pos, inv_freq, q, k, q_out, k_out, stream):
    """Checked arguments of both rotating calls, their outputs allocated unless given:
    (rows, q_out, k_out, (q, stride, out, stride), (heads of k, k, stride, out, stride))."""
    rows, Hq = q.shape[0], q.shape[1]
    if pos.dtype != torch.int32 or pos.shape != (rows,) or not pos.is_contiguous():
        raise ValueError("pos: contiguous int32 [rows] expected")
    if inv_freq.dtype != torch.float32 or not inv_freq.is_contiguous():
        raise ValueError("inv_freq: contiguous fp32 expected")
    if q_out is None:
        q_out = _new(stream, (rows, Hq, q.shape[2]), q.dtype, q.device)
    if k is not None and k_out is None:
        k_out = _new(stream, k.shape, k.dtype, k.device)
    if q_out.shape != q.shape or (k is not None and (k_out.shape != k.shape or k.shape[0] != rows)):
        raise ValueError("%s: outputs shaped as their inputs expected" % what)
    ka = (0, None, 0, None, 0) if k is None else (
        k.shape[1], *_rows(k, "k", L.head_dim), *_rows(k_out, "k_out", L.head_dim))
    qa = (*_rows(q, "q", L.head_dim), *_rows(q_out, "q_out", L.head_dim))
    return rows, q_out, k_out, qa, ka


def rotate(L, pos, inv_freq, q, k=None, style=ROPE_HALF, scale=1.0, q_out=None, k_out=None, stream=None):
    """Rotary positions: q fp16 [rows, Hq, D], k fp16 [rows, Hkv, D] or None (rows may be strided), pos int32
    [rows], inv_freq fp32 [rot_dim / 2] (device) -> (q_out, k_out), contiguous unless given; q_out=q turns in
    place."""
    rows, q_out, k_out, qa, (Hkv, kp, ks, kop, kos) = _rotate_args(
        "rotate", L, pos, inv_freq, q, k, q_out, k_out, stream)
    _on_one_gpu("rotate", q, k, pos, inv_freq, q_out, k_out)
    _check(lib().diffkv_rotate(C.byref(L), rows, _ptr(pos), _ptr(inv_freq), 2 * inv_freq.shape[0], int(style),
                               float(scale), q.shape[1], *qa, Hkv, kp, ks, kop, kos, _stream(stream)),
           "diffkv_rotate")
    return q_out, k_out


def norm_rotate(L, pos, inv_freq, q, k=None, q_weight=None, k_weight=None, eps=1e-6, style=ROPE_HALF, scale=1.0,
                q_out=None, k_out=None, stream=None):
    """Each head over its root mean square times its side's weights (fp32 [D] or None: ones), then rotated:
    arguments and results as rotate."""
    at = _stream_at("norm_rotate", stream, q)
    rows, q_out, k_out, (qp, qs, qop, qos), (Hkv, kp, ks, kop, kos) = _rotate_args(
        "norm_rotate", L, pos, inv_freq, q, k, q_out, k_out, stream)
    _dense(q_weight, "q_weight", torch.float32, L.head_dim)
    _dense(k_weight, "k_weight", torch.float32, L.head_dim)
    _on_one_gpu("norm_rotate", q, k, pos, inv_freq, q_weight, k_weight, q_out, k_out)
    _check(lib().diffkv_norm_rotate(C.byref(L), rows, _ptr(pos), _ptr(inv_freq), 2 * inv_freq.shape[0], int(style),
                                    float(scale), float(eps), q.shape[1], qp, qs, _ptr(q_weight), qop, qos, Hkv, kp, ks,
                                    _ptr(k_weight), kop, kos, at), "diffkv_norm_rotate")
    return q_out, k_out


def _chunk(cache, new_len, max_new, what, stream, q, *rows):
    if new_len.dtype != torch.int32 or new_len.shape != (cache.num_seqs,) or not new_len.is_contiguous():
        raise ValueError("%s: new_len: contiguous int32 [num_seqs] expected" % what)
    if max_new is None:
        max_new = _longest(new_len, stream)
    for t in rows:
        if t.shape[0] != q.shape[0] or t.shape[1] != cache.num_kv_heads:
            raise ValueError("%s: [rows, num_kv_heads, head_dim] keys and values expected" % what)
    return int(max_new)


def _dense(t, what, dtype, *shape):
    if t is not None and (t.dtype != dtype or t.shape != shape or not t.is_contiguous()):
        raise ValueError("%s: contiguous %s %s expected" % (what, dtype, list(shape)))


def chunk_attention(cache, new_len, q, k, v, sm_scale, cap=0.0, window=0, slopes=None, out=None, lse=None,
                    max_new=None, ws=None, stream=None, want_lse=True):
    """diffkv_chunk_attention: q fp16 [rows, Hq, D], k, v fp16 [rows, Hkv, D] (device, rows concatenated per
    sequence, may be strided), new_len int32 [B] (device) -> out fp16 [rows, Hq, D], lse fp32 [rows, Hq].
    Call it before the rows are appended."""
    rows, Hq, D = q.shape
    max_new = _chunk(cache, new_len, max_new, "chunk_attention", stream, q, k, v)
    if out is None:
        out = _new(stream, (rows, Hq, D), torch.float16, q.device)
    if lse is None and want_lse:
        lse = _new(stream, (rows, Hq), torch.float32, q.device)
    _dense(out, "out", torch.float16, rows, Hq, D)
    _dense(lse, "lse", torch.float32, rows, Hq)
    _dense(slopes, "slopes", torch.float32, Hq)
    sizes = (OP_CHUNK_ATTENTION, cache.L, cache.num_seqs, Hq, cache.num_kv_heads, rows)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), q.device, stream)
    (qp, qs), (kp, ks), (vp, vs) = (_rows(t, w, cache.L.head_dim) for t, w in ((q, "q"), (k, "k"), (v, "v")))
    _on_one_gpu("chunk_attention", q, k, v, new_len, slopes, out, lse, ws)
    _check_ws(lib().diffkv_chunk_attention(
        C.byref(cache.L), _cache_struct(cache), rows, max_new, _ptr(new_len), Hq, qp, qs, kp, ks, vp, vs,
        float(sm_scale), _form(cap, window, slopes), _ptr(out), _ptr(lse), ws.data_ptr(), ws.nbytes, _stream(stream)),
        "diffkv_chunk_attention", *sizes)
    return out, lse


def chunk_significance(cache, new_len, q, k, sm_scale, lse, cap=0.0, window=0, slopes=None, score=None,
                       max_new=None, ws=None, stream=None):
    """diffkv_chunk_significance: the chunk's probabilities (lse from chunk_attention with the same q, k and
    form) enter the cached tokens' scores in place; returns the new tokens' scores, fp32 [rows, Hkv]."""
    rows, Hq = q.shape[0], q.shape[1]
    max_new = _chunk(cache, new_len, max_new, "chunk_significance", stream, q, k)
    if score is None:
        score = _new(stream, (rows, cache.num_kv_heads), torch.float32, q.device)
    _dense(lse, "lse", torch.float32, rows, Hq)
    _dense(score, "score", torch.float32, rows, cache.num_kv_heads)
    _dense(slopes, "slopes", torch.float32, Hq)
    sizes = (OP_CHUNK_SIGNIFICANCE, cache.L, cache.num_seqs, Hq, cache.num_kv_heads, rows)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), q.device, stream)
    (qp, qs), (kp, ks) = (_rows(t, w, cache.L.head_dim) for t, w in ((q, "q"), (k, "k")))
    _on_one_gpu("chunk_significance", q, k, new_len, slopes, lse, score, ws)
    _check_ws(lib().diffkv_chunk_significance(
        C.byref(cache.L), _cache_struct(cache), rows, max_new, _ptr(new_len), Hq, qp, qs, kp, ks, float(sm_scale),
        _form(cap, window, slopes), _ptr(lse), _ptr(score), ws.data_ptr(), ws.nbytes, _stream(stream)),
        "diffkv_chunk_significance", *sizes)
    return score


class BlockCache:
    """Device tensors of one uniform 8-bit cache (diffkv_block_cache); the library owns none of them.  `table` int32
    [num_seqs, ceil(max_seq_len / 32)] (block IDs, -1: not kept) and `seq_len` int32 [num_seqs] are the program's to
    write.  `buffers`: (pool, scale, table, tail, seq_len, status) to use instead of new ones (caches of a model's
    layers share table and seq_len).  The tensors are the handle's for its life: their contents may be written, but
    others need another handle."""

    def __init__(self, L, num_blocks, num_seqs, num_kv_heads, fmt=BLOCK_E4M3, device="cuda", buffers=None):
        self.L = L
        self.num_blocks, self.num_seqs, self.num_kv_heads = int(num_blocks), int(num_seqs), int(num_kv_heads)
        self.fmt = int(fmt)
        width = -(-L.max_seq_len // BLOCK_TOKENS)
        D = L.head_dim
        if buffers is None:
            dev = torch.device(device)
            z = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device=dev)
            buffers = (z(self.num_blocks, self.num_kv_heads, 2, BLOCK_TOKENS * D, dtype=torch.uint8),
                       torch.ones((self.num_blocks, self.num_kv_heads, 2), dtype=torch.float32, device=dev),
                       torch.full((self.num_seqs, width), -1, dtype=torch.int32, device=dev),
                       z(self.num_seqs, self.num_kv_heads, 2, BLOCK_TOKENS, D, dtype=torch.float16),
                       z(self.num_seqs, dtype=torch.int32), z(1, dtype=torch.int32))
        self._tensors = tuple(buffers)
        pool, scale, table, tail, seq_len, status = self._tensors
        for t, what, dtype, shape in (
                (pool, "pool", torch.uint8, (self.num_blocks, self.num_kv_heads, 2, BLOCK_TOKENS * D)),
                (scale, "scale", torch.float32, (self.num_blocks, self.num_kv_heads, 2))):
            if t.dtype != dtype or not t.is_contiguous() or t.shape[0] < shape[0] or t.shape[1:] != shape[1:]:
                raise ValueError("%s: contiguous %s %s expected" % (what, dtype, list(shape)))
        _dense(table, "table", torch.int32, self.num_seqs, width)
        _dense(tail, "tail", torch.float16, self.num_seqs, self.num_kv_heads, 2, BLOCK_TOKENS, D)
        _dense(seq_len, "seq_len", torch.int32, self.num_seqs)
        _dense(status, "status", torch.int32, 1)
        if any(t.device != pool.device for t in self._tensors):
            raise ValueError("BlockCache: tensors on one device expected")
        self._struct = BlockCacheStruct(pool.data_ptr(), scale.data_ptr(), self.num_blocks, table.data_ptr(),
                                        tail.data_ptr(), seq_len.data_ptr(), status.data_ptr(), self.num_seqs,
                                        self.num_kv_heads, self.fmt)

    def _same(self, i, t):  # (what `cache.seq_len += n` ends with)
        if t is not self._tensors[i]:
            raise AttributeError("a BlockCache's tensors are its handle's for life: write into them, or make another")

    pool, scale, table, tail, seq_len, status = (
        property(lambda self, i=i: self._tensors[i], lambda self, t, i=i: self._same(i, t)) for i in range(6))

    def tensors(self):
        return self._tensors

    def struct(self):
        return self._struct


def _block_lens(cache, t, what):
    if t.dtype != torch.int32 or t.shape != (cache.num_seqs,) or not t.is_contiguous():
        raise ValueError("%s: lengths: contiguous int32 [num_seqs] expected" % what)


def _block_rows(cache, k, v, what, rows):
    """Addresses and row strides of keys and values [rows, num_kv_heads, head_dim]."""
    D = cache.L.head_dim
    kp, ks = _rows(k, "k", D)
    vp, vs = _rows(v, "v", D)
    if k.shape != (rows, cache.num_kv_heads, D) or v.shape != k.shape:
        raise ValueError("%s: [rows, num_kv_heads, head_dim] keys and values expected" % what)
    return kp, ks, vp, vs


def block_append(cache, new_len, k, v, max_new=None, stream=None):
    """diffkv_block_append: k, v fp16 [rows, Hkv, D] (device, rows concatenated per sequence, may be strided), new_len
    int32 [B] (device), into cache (a BlockCache) at seq_len, which is not advanced."""
    _block_lens(cache, new_len, "block_append")
    rows = k.shape[0]
    kv = _block_rows(cache, k, v, "block_append", rows)
    _on_one_gpu("block_append", k, v, new_len, cache.pool)
    at = _stream_at("block_append", stream, k)
    if max_new is None:
        max_new = _longest(new_len, stream)
    _check(lib().diffkv_block_append(cache.L, cache.struct(), rows, int(max_new), new_len.data_ptr(), *kv, at),
           "diffkv_block_append")


def block_read(cache, start, count, total, max_count=None, k_out=None, v_out=None, stream=None):
    """diffkv_block_read: positions start[b] .. + count[b] - 1 of each sequence (int32 [B], device) as fp16 rows
    [total, Hkv, D], one sequence's behind the other's -> (k_out, v_out)."""
    shape = (int(total), cache.num_kv_heads, cache.L.head_dim)
    at = _stream_at("block_read", stream, cache.pool)
    k_out, v_out = (_new(stream, shape, torch.float16, cache.tail.device) if t is None else t
                    for t in (k_out, v_out))
    _block_lens(cache, start, "block_read")
    _block_lens(cache, count, "block_read")
    kv = _block_rows(cache, k_out, v_out, "block_read", shape[0])
    _on_one_gpu("block_read", k_out, v_out, start, count, cache.pool)
    if max_count is None:
        max_count = _longest(count, stream)
    _check(lib().diffkv_block_read(cache.L, cache.struct(), shape[0], int(max_count), start.data_ptr(), count.data_ptr(), *kv, at),
           "diffkv_block_read")
    return k_out, v_out


def block_attention(cache, new_len, q, k, v, sm_scale, cap=0.0, window=0, sinks=0, slopes=None, out=None, lse=None,
                    max_new=None, ws=None, stream=None, want_lse=True):
    """diffkv_block_attention: q fp16 [rows, Hq, D], k, v fp16 [rows, Hkv, D] (device, rows concatenated per sequence,
    may be strided), new_len int32 [B] (device) over cache (a BlockCache) -> out fp16 [rows, Hq, D], lse fp32
    [rows, Hq].  With a window the first `sinks` tokens stay visible.  Call it before the rows are appended."""
    rows, Hq, D = q.shape
    _block_lens(cache, new_len, "block_attention")
    kv = _block_rows(cache, k, v, "block_attention", rows)
    qp, qs = _rows(q, "q", cache.L.head_dim)
    at = _stream_at("block_attention", stream, cache.pool)
    if out is None:
        out = _new(stream, (rows, Hq, D), torch.float16, q.device)
    if lse is None and want_lse:
        lse = _new(stream, (rows, Hq), torch.float32, q.device)
    _dense(out, "out", torch.float16, rows, Hq, D)
    _dense(lse, "lse", torch.float32, rows, Hq)
    _dense(slopes, "slopes", torch.float32, Hq)
    sizes = (OP_BLOCK_ATTENTION, cache.L, cache.num_seqs, Hq, cache.num_kv_heads, rows)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), q.device, stream)
    _on_one_gpu("block_attention", q, k, v, new_len, slopes, out, lse, ws, cache.pool)
    if max_new is None:
        max_new = _longest(new_len, stream)
    _check_ws(lib().diffkv_block_attention(
        cache.L, cache.struct(), rows, int(max_new), new_len.data_ptr(), Hq, qp, qs, *kv, float(sm_scale),
        _form(cap, window, slopes), int(sinks), out.data_ptr(), _ptr(lse), ws.data_ptr(), ws.nbytes, at),
        "diffkv_block_attention", *sizes)
    return out, lse


def compact_free_list(cache, release, num_tables=None, ws=None, stream=None):
    """release uint8 [num_tables, p_max] (device)."""
    L = cache.L
    nt = cache.num_tables if num_tables is None else num_tables
    sizes = (OP_COMPACT, L, cache.num_seqs, 0, cache.num_kv_heads)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), cache.pool.device, stream)
    _check_ws(lib().diffkv_compact_free_list(C.byref(L), _cache_struct(cache), int(nt), _ptr(release), ws.data_ptr(), ws.nbytes,
                       _stream(stream)), "diffkv_compact_free_list", *sizes)
    return ws


def alloc_pages(cache, demand, num_tables=None, ws=None, stream=None):
    """demand int32 [num_tables, 2] (device)."""
    L = cache.L
    nt = cache.num_tables if num_tables is None else num_tables
    sizes = (OP_ALLOC, L, cache.num_seqs, 0, cache.num_kv_heads)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), cache.pool.device, stream)
    _check_ws(lib().diffkv_alloc_pages(C.byref(L), _cache_struct(cache), int(nt), _ptr(demand), ws.data_ptr(), ws.nbytes,
                       _stream(stream)), "diffkv_alloc_pages", *sizes)
    return ws


def generation_step(cache, alpha_h, alpha_l, recent_window, ws=None, stream=None):
    """One decode step's generation-phase policy for every table (Algorithm 1)."""
    L = cache.L
    sizes = (OP_GENERATION, L, cache.num_seqs, 0, cache.num_kv_heads)
    if ws is None:
        ws = _new_ws(workspace_size(*sizes), cache.pool.device, stream)
    _check_ws(lib().diffkv_generation_step(C.byref(L), _cache_struct(cache), float(alpha_h), float(alpha_l),
                                           int(recent_window), ws.data_ptr(), ws.nbytes, _stream(stream)),
              "diffkv_generation_step", *sizes)
    return ws
