"""Thin ctypes binding of the HIP codec library (include/zc.h).

Argument marshalling only: every step of the codec runs in the library's
kernels.  PyTorch supplies device memory and the current stream.  There is no
fallback: if libzc.so is not built (see __graft_entry__.build) importing the
library handle raises.
"""
import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libzc.so")

FMT_BF16, FMT_FP8_E4M3, FMT_FP4_E2M1_MX, FMT_FP8_E4M3_BYTES, FMT_FP4_E2M1_MX_BYTES, FMT_FP4_E2M1_NV, FMT_FP8_E5M2 = 1, 2, 3, 4, 5, 6, 7
POLICY_HUFF_ALL, POLICY_AUTO = 0, 1
FLAG_HOST_CODES = 1
FLAG_REVERSE_FIELDS = 2
NOALLOC_SCRATCH_BYTES = 4 << 20
MODE_EMPTY, MODE_HUFF, MODE_RAW, MODE_CONST = 0, 1, 2, 3
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_BUFFER_TOO_SMALL, ERR_CORRUPT, ERR_DEVICE = range(6)

EXPORTS = ["zc_compress_bound", "zc_workspace_bytes", "zc_compress", "zc_compress_batch", "zc_read_info",
           "zc_decompress", "zc_decompress_chunks", "zc_decompress_batch", "zc_decompress_batch_plan",
           "zc_decompress_batch_run", "zc_stats", "zc_build_code", "zc_train_code", "zc_compress_with_code",
           "zc_compress_batch_with_code", "zc_compress_batch_with_code_async", "zc_compress_batch_async", "zc_code_stale",
           "zc_validate_container", "zc_release_host_buffers", "zc_compress_noalloc", "zc_copy_reference", "zc_status_string",
           "zc_attend", "zc_attend_shared", "zc_attend_workspace_bytes", "zc_evict", "zc_kv_write", "zc_kv_read"]


class Params(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("format", C.c_uint32), ("chunk_bytes", C.c_uint32),
                ("max_code_len", C.c_uint32 * 3), ("streams_per_chunk", C.c_uint32), ("policy", C.c_uint32),
                ("flags", C.c_uint32)]


class Info(C.Structure):
    _fields_ = [("format", C.c_uint32), ("policy", C.c_uint32), ("streams", C.c_uint32), ("n_fields", C.c_uint32),
                ("xor_delta", C.c_uint32), ("chunk_bytes", C.c_uint32), ("n_chunks", C.c_uint32), ("payload_order", C.c_uint32),
                ("n_elems", C.c_uint64), ("total_bytes", C.c_uint64), ("payload_offset", C.c_uint64),
                ("table_offset", C.c_uint64 * 3), ("index_offset", C.c_uint64 * 3),
                ("mode", C.c_uint8 * 3), ("sym_bits", C.c_uint8 * 3), ("max_len", C.c_uint8 * 3), ("const_symbol", C.c_uint8 * 3),
                ("code_len", (C.c_uint8 * 256) * 3)]


class FieldStats(C.Structure):
    _fields_ = [("alphabet", C.c_uint32), ("distinct", C.c_uint32), ("mode", C.c_uint32), ("max_len", C.c_uint32),
                ("n_symbols", C.c_uint64), ("hist", C.c_uint64 * 256), ("code_len", C.c_uint8 * 256),
                ("entropy_bits", C.c_double), ("mean_code_len", C.c_double), ("payload_bits", C.c_uint64),
                ("stream_bytes", C.c_uint64), ("ratio_payload", C.c_double)]


class StatsOut(C.Structure):
    _fields_ = [("n_fields", C.c_uint32), ("reserved", C.c_uint32), ("raw_bytes", C.c_uint64),
                ("container_bytes", C.c_uint64), ("ratio_payload_total", C.c_double),
                ("ratio_container_total", C.c_double), ("field", FieldStats * 3)]


class Tensor(C.Structure):
    _fields_ = [("d_src", C.c_void_p), ("d_xor_base", C.c_void_p), ("d_scales", C.c_void_p), ("n_elems", C.c_uint64),
                ("d_comp", C.c_void_p), ("comp_capacity", C.c_uint64), ("d_dst", C.c_void_p), ("d_scales_out", C.c_void_p),
                ("d_chunk_ids", C.c_void_p), ("n_chunk_ids", C.c_uint32), ("reserved", C.c_uint32),
                ("out_bytes", C.c_uint64), ("info", Info)]


class BatchPlan(C.Structure):
    _fields_ = [("format", C.c_uint32), ("streams", C.c_uint32), ("n_tensors", C.c_uint32), ("n_fast_work", C.c_uint32),
                ("n_work", C.c_uint32), ("fast_kernel", C.c_uint32), ("fast_exp_kind", C.c_uint32), ("fast_sm_kind", C.c_uint32),
                ("n_rings", C.c_uint32), ("xor_delta", C.c_uint32), ("scattered", C.c_uint32), ("tail_kernel", C.c_uint32),
                ("fast_work_offset", C.c_uint64), ("work_offset", C.c_uint64)]


class KvCache(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("format", C.c_uint32), ("n_seqs", C.c_uint32), ("n_heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("page_tokens", C.c_uint32), ("table_pages", C.c_uint32), ("n_pages", C.c_uint32),
                ("d_k_pages", C.c_void_p), ("d_v_pages", C.c_void_p), ("d_table", C.c_void_p), ("d_lengths", C.c_void_p),
                ("d_k_scales", C.c_void_p), ("d_v_scales", C.c_void_p), ("d_k_block_scales", C.c_void_p), ("d_v_block_scales", C.c_void_p)]


class KvRows(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_tokens", C.c_uint32), ("d_k", C.c_void_p), ("d_v", C.c_void_p),
                ("k_token_stride", C.c_uint64), ("k_head_stride", C.c_uint64), ("v_token_stride", C.c_uint64), ("v_head_stride", C.c_uint64),
                ("d_q_start", C.c_void_p)]


class AttendArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_tokens", C.c_uint32), ("n_q_heads", C.c_uint32), ("max_q_len", C.c_uint32),
                ("window", C.c_uint32), ("sinks", C.c_uint32), ("max_kv_len", C.c_uint32), ("max_prefix_len", C.c_uint32),
                ("scale", C.c_float), ("reserved", C.c_uint32), ("d_q", C.c_void_p), ("d_out", C.c_void_p),
                ("q_token_stride", C.c_uint64), ("q_head_stride", C.c_uint64), ("out_token_stride", C.c_uint64), ("out_head_stride", C.c_uint64),
                ("d_q_start", C.c_void_p), ("d_lse", C.c_void_p), ("d_weights_in", C.c_void_p), ("d_weights_out", C.c_void_p)]


_ATTEND_ARGS_BYTES = C.sizeof(AttendArgs)
_KV_ROWS_BYTES = C.sizeof(KvRows)
# The members in their order: a structure made of packed bytes takes half the time of one whose members are set one by one (0.9 us, of calls of 10).
_pack_attend_args = struct.Struct("=8IfI10Q").pack
_pack_kv_rows = struct.Struct("=2I7Q").pack


class ZcError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        RuntimeError.__init__(self, "%s: %s" % (what, status_string(status)))


_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("%s is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        vp, u64, u32 = C.c_void_p, C.c_uint64, C.c_uint32
        L.zc_status_string.restype = C.c_char_p
        L.zc_status_string.argtypes = [C.c_int]
        L.zc_compress_bound.restype = u64
        L.zc_compress_bound.argtypes = [u64, C.POINTER(Params)]
        L.zc_workspace_bytes.restype = u64
        L.zc_workspace_bytes.argtypes = [C.POINTER(u64), u32, C.POINTER(Params)]
        L.zc_compress.restype = C.c_int
        L.zc_compress.argtypes = [vp, u64, C.POINTER(Params), vp, vp, vp, u64, C.POINTER(u64), C.POINTER(Info), vp, u64, vp]
        L.zc_compress_batch.restype = C.c_int
        L.zc_compress_batch.argtypes = [C.POINTER(Tensor), u32, C.POINTER(Params), vp, u64, vp]
        L.zc_compress_noalloc.restype = C.c_int
        L.zc_compress_noalloc.argtypes = [vp, u64, C.POINTER(Params), vp, vp, vp, u64, vp]
        L.zc_copy_reference.restype = C.c_int
        L.zc_copy_reference.argtypes = [vp, vp, u64, u32, vp]
        L.zc_code_stale.restype = C.c_int
        L.zc_code_stale.argtypes = [C.POINTER(Info), C.POINTER(Info), C.c_double]
        L.zc_train_code.restype = C.c_int
        L.zc_train_code.argtypes = [vp, u64, C.POINTER(Params), vp, vp, C.POINTER(Info), vp, u64, vp]
        L.zc_compress_with_code.restype = C.c_int
        L.zc_compress_with_code.argtypes = [vp, u64, C.POINTER(Params), C.POINTER(Info), vp, vp, vp, u64, C.POINTER(u64), C.POINTER(Info), vp, u64, vp]
        L.zc_compress_batch_with_code.restype = C.c_int
        L.zc_compress_batch_with_code.argtypes = [C.POINTER(Tensor), u32, C.POINTER(Params), C.POINTER(Info), vp, u64, vp]
        L.zc_compress_batch_with_code_async.restype = C.c_int
        L.zc_compress_batch_with_code_async.argtypes = [C.POINTER(Tensor), u32, C.POINTER(Params), C.POINTER(Info), vp, u64, vp]
        L.zc_compress_batch_async.restype = C.c_int
        L.zc_compress_batch_async.argtypes = [C.POINTER(Tensor), u32, C.POINTER(Params), vp, u64, vp]
        L.zc_read_info.restype = C.c_int
        L.zc_read_info.argtypes = [vp, u64, C.c_int, C.POINTER(Info), vp]
        L.zc_decompress.restype = C.c_int
        L.zc_decompress.argtypes = [vp, u64, C.POINTER(Info), vp, u64, vp, vp, vp]
        L.zc_decompress_chunks.restype = C.c_int
        L.zc_decompress_chunks.argtypes = [vp, u64, C.POINTER(Info), vp, u32, vp, u64, vp, vp, vp]
        L.zc_decompress_batch.restype = C.c_int
        L.zc_decompress_batch.argtypes = [C.POINTER(Tensor), u32, vp, u64, vp]
        L.zc_decompress_batch_plan.restype = C.c_int
        L.zc_decompress_batch_plan.argtypes = [C.POINTER(Tensor), u32, vp, u64, C.POINTER(BatchPlan), vp]
        L.zc_decompress_batch_run.restype = C.c_int
        L.zc_decompress_batch_run.argtypes = [C.POINTER(BatchPlan), vp, vp]
        L.zc_stats.restype = C.c_int
        L.zc_stats.argtypes = [vp, u64, C.POINTER(Params), vp, vp, C.POINTER(StatsOut), vp, u64, vp]
        L.zc_validate_container.restype = C.c_int
        L.zc_validate_container.argtypes = [vp, u64, u64, C.c_int, C.POINTER(Info)]
        L.zc_release_host_buffers.restype = C.c_int
        L.zc_release_host_buffers.argtypes = []
        L.zc_attend_workspace_bytes.restype = u64
        L.zc_attend_workspace_bytes.argtypes = [C.POINTER(AttendArgs), C.POINTER(KvCache), C.POINTER(KvCache)]
        L.zc_attend.restype = C.c_int
        L.zc_attend.argtypes = [C.POINTER(AttendArgs), C.POINTER(KvCache), vp, u64, vp]
        L.zc_attend_shared.restype = C.c_int
        L.zc_attend_shared.argtypes = [C.POINTER(AttendArgs), C.POINTER(KvCache), C.POINTER(KvCache), vp, u64, vp]
        L.zc_evict.restype = C.c_int
        L.zc_evict.argtypes = [C.POINTER(KvCache), vp, u32, u32, u32, C.POINTER(KvCache), vp, vp, vp]
        for call in (L.zc_kv_write, L.zc_kv_read):
            call.restype = C.c_int
            call.argtypes = [C.POINTER(KvRows), C.POINTER(KvCache), vp]
        L.zc_build_code.restype = C.c_int
        L.zc_build_code.argtypes = [C.POINTER(u64), u32, u32, C.POINTER(C.c_uint8), C.POINTER(C.c_uint16)]
        _lib = L
    return _lib


def status_string(status):
    return lib().zc_status_string(status).decode()


def params(fmt, chunk_bytes, max_code_len=(0, 0, 0), streams=0, policy=POLICY_HUFF_ALL, flags=0):
    p = Params()
    p.struct_size = C.sizeof(Params)
    p.format, p.chunk_bytes, p.streams_per_chunk, p.policy, p.flags = fmt, chunk_bytes, streams, policy, flags
    for i in range(3):
        p.max_code_len[i] = max_code_len[i]
    return p


def elem_bits(fmt):
    return {FMT_BF16: 16, FMT_FP8_E4M3: 8, FMT_FP4_E2M1_MX: 4, FMT_FP8_E4M3_BYTES: 8, FMT_FP4_E2M1_MX_BYTES: 4, FMT_FP4_E2M1_NV: 4, FMT_FP8_E5M2: 8}[fmt]


def scale_block(fmt):
    """Elements that share one scale byte (0: the format has none)."""
    return {FMT_FP4_E2M1_MX: 32, FMT_FP4_E2M1_MX_BYTES: 32, FMT_FP4_E2M1_NV: 16}.get(fmt, 0)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(status, what):
    if status != OK:
        raise ZcError(status, what)


def compress_bound(n_elems, p):
    return int(lib().zc_compress_bound(n_elems, C.byref(p)))


def workspace_bytes(n_elems_list, p):
    arr = (C.c_uint64 * len(n_elems_list))(*n_elems_list)
    return int(lib().zc_workspace_bytes(arr, len(n_elems_list), C.byref(p)))


def build_code(hist, limit):
    """Host-only: (lengths, codes) of the library's code construction for a histogram."""
    n = len(hist)
    h = (C.c_uint64 * n)(*[int(v) for v in hist])
    ln = (C.c_uint8 * n)()
    cd = (C.c_uint16 * n)()
    _check(lib().zc_build_code(h, n, limit, ln, cd), "zc_build_code")
    return list(ln), list(cd)


def _workspace(n_elems_list, p, device):
    need = workspace_bytes(n_elems_list, p)
    if need == 0:
        raise ZcError(ERR_INVALID_ARG, "zc_workspace_bytes")
    return torch.empty(need, dtype=torch.uint8, device=device)


def compress(src, n_elems, p, xor_base=None, scales=None, dst=None, ws=None):
    """src/xor_base/scales/dst/ws: CUDA tensors (any dtype, contiguous).  Returns (container view, Info)."""
    dev = src.device
    if dst is None:
        dst = torch.empty(max(compress_bound(n_elems, p), 16), dtype=torch.uint8, device=dev)
    if ws is None:
        ws = _workspace([n_elems], p, dev)
    size = C.c_uint64(0)
    info = Info()
    st = lib().zc_compress(_ptr(src), n_elems, C.byref(p), _ptr(xor_base), _ptr(scales), _ptr(dst), dst.numel() * dst.element_size(),
                           C.byref(size), C.byref(info), _ptr(ws), ws.numel(), _stream())
    _check(st, "zc_compress")
    return dst.view(torch.uint8).reshape(-1)[:size.value], info


def compress_noalloc(src, n_elems, p, dst, xor_base=None, scales=None):
    """Queue the compression of one tensor into dst (at least compress_bound bytes) without a workspace and
    without any allocation; the container's size is in its header once the stream gets there (read_info)."""
    st = lib().zc_compress_noalloc(_ptr(src), n_elems, C.byref(p), _ptr(xor_base), _ptr(scales), _ptr(dst),
                                   dst.numel() * dst.element_size(), _stream())
    _check(st, "zc_compress_noalloc")


def train_code(src, n_elems, p, xor_base=None, scales=None, ws=None):
    """Static dictionary (an Info whose mode/code_len fields are meaningful) from a representative tensor."""
    if ws is None:
        ws = _workspace([n_elems], p, src.device)
    code = Info()
    st = lib().zc_train_code(_ptr(src), n_elems, C.byref(p), _ptr(xor_base), _ptr(scales), C.byref(code), _ptr(ws), ws.numel(), _stream())
    _check(st, "zc_train_code")
    return code


def code_stale(code, written, slack=0.02):
    """Refresh test for a static dictionary: True when `written` (the Info of a compress_with_code call) is
    larger relative to its raw size than the training tensor was, by more than `slack`."""
    r = lib().zc_code_stale(C.byref(code), C.byref(written), slack)
    if r < 0:
        raise ZcError(ERR_INVALID_ARG, "zc_code_stale")
    return bool(r)


def compress_with_code(src, n_elems, p, code, xor_base=None, scales=None, dst=None, ws=None):
    dev = src.device
    if dst is None:
        dst = torch.empty(max(compress_bound(n_elems, p), 16), dtype=torch.uint8, device=dev)
    if ws is None:
        ws = _workspace([n_elems], p, dev)
    size = C.c_uint64(0)
    info = Info()
    st = lib().zc_compress_with_code(_ptr(src), n_elems, C.byref(p), C.byref(code), _ptr(xor_base), _ptr(scales), _ptr(dst),
                                     dst.numel() * dst.element_size(), C.byref(size), C.byref(info), _ptr(ws), ws.numel(), _stream())
    _check(st, "zc_compress_with_code")
    return dst.view(torch.uint8).reshape(-1)[:size.value], info


def read_info(comp, check_index=False):
    info = Info()
    _check(lib().zc_read_info(_ptr(comp), comp.numel(), 1 if check_index else 0, C.byref(info), _stream()), "zc_read_info")
    return info


def validate_container(host_bytes, check_index=True, container_bytes=None):
    """Host only: validate a container held in host memory (bytes, bytearray or a numpy uint8 array); returns its
    Info.  container_bytes: size of the whole container when host_bytes is only its beginning."""
    buf = (C.c_uint8 * len(host_bytes)).from_buffer_copy(bytes(host_bytes))
    info = Info()
    total = len(host_bytes) if container_bytes is None else container_bytes
    _check(lib().zc_validate_container(buf, len(host_bytes), total, 1 if check_index else 0, C.byref(info)), "zc_validate_container")
    return info


def copy_reference(src, dst, chunk_bytes=0):
    """Queue the library's plain copy kernel (the bandwidth yardstick) from src to dst, both CUDA tensors of equal size;
    chunk_bytes != 0: one wavefront per chunk, as the 64-lane codec kernels walk through memory."""
    _check(lib().zc_copy_reference(_ptr(src), _ptr(dst), src.numel() * src.element_size(), chunk_bytes, _stream()), "zc_copy_reference")


def release_host_buffers():
    _check(lib().zc_release_host_buffers(), "zc_release_host_buffers")


def decompress(comp, info=None, out=None, scales_out=None, xor_base=None, read_header_in_call=False):
    """Returns (elements as uint8 tensor, scales or None).  read_header_in_call: pass no Info to the library, which
    then reads the header itself (a blocking copy) before it queues the decode."""
    if info is None:
        info = read_info(comp)
    raw = (info.n_elems * elem_bits(info.format) + 7) // 8
    if out is None:
        out = torch.empty(raw, dtype=torch.uint8, device=comp.device)
    if info.n_fields == 3 and scales_out is None:
        scales_out = torch.empty(max(info.n_elems // scale_block(info.format), 1), dtype=torch.uint8, device=comp.device)
    st = lib().zc_decompress(_ptr(comp), comp.numel(), None if read_header_in_call else C.byref(info), _ptr(out),
                             out.numel() * out.element_size(), _ptr(scales_out), _ptr(xor_base), _stream())
    _check(st, "zc_decompress")
    return out, scales_out


def decompress_chunks(comp, info, ids, out=None, scales_out=None, xor_base=None):
    """ids: int32/uint32 CUDA tensor of chunk ids; chunk ids[i] lands at out[i*chunk_bytes:]."""
    n = ids.numel()
    if out is None:
        out = torch.empty(n * info.chunk_bytes, dtype=torch.uint8, device=comp.device)
    if info.n_fields == 3 and scales_out is None:
        scales_out = torch.empty(max(n * info.chunk_bytes * 2 // scale_block(info.format), 1), dtype=torch.uint8, device=comp.device)
    st = lib().zc_decompress_chunks(_ptr(comp), comp.numel(), C.byref(info), _ptr(ids), n, _ptr(out),
                                    out.numel() * out.element_size(), _ptr(scales_out), _ptr(xor_base), _stream())
    _check(st, "zc_decompress_chunks")
    return out, scales_out


def stats(src, n_elems, p, xor_base=None, scales=None, ws=None):
    if ws is None:
        ws = _workspace([n_elems], p, src.device)
    out = StatsOut()
    st = lib().zc_stats(_ptr(src), n_elems, C.byref(p), _ptr(xor_base), _ptr(scales), C.byref(out), _ptr(ws), ws.numel(), _stream())
    _check(st, "zc_stats")
    return out


class Batch:
    """A set of tensors compressed / decompressed with one launch sequence.

    Holds the host array of zc_tensor descriptors plus the torch tensors that own the
    device memory, so that repeated calls allocate nothing."""

    def __init__(self, srcs, n_elems, p, xor_bases=None, scales=None):
        self.p = p
        self.n = len(srcs)
        self.srcs, self.bases, self.scales = list(srcs), xor_bases, scales
        dev = srcs[0].device
        self.arr = (Tensor * self.n)()
        self.caps = [max(compress_bound(n, p), 16) for n in n_elems]
        # one arena for all containers, each slot 256-byte aligned
        offs, total = [], 0
        for c in self.caps:
            offs.append(total)
            total += (c + 255) // 256 * 256
        self.arena = torch.empty(total, dtype=torch.uint8, device=dev)
        self.comp = [self.arena[o:o + c] for o, c in zip(offs, self.caps)]
        self.ws = _workspace(list(n_elems), p, dev)
        # the decode plan lives in a workspace of its own: compress() rewrites self.ws
        self.ws_plan = torch.empty(self.ws.numel(), dtype=torch.uint8, device=dev)
        for i in range(self.n):
            a = self.arr[i]
            a.d_src = srcs[i].data_ptr()
            a.d_xor_base = xor_bases[i].data_ptr() if xor_bases else None
            a.d_scales = scales[i].data_ptr() if scales else None
            a.n_elems = n_elems[i]
            a.d_comp = self.comp[i].data_ptr()
            a.comp_capacity = self.caps[i]
        self.out = None
        self.scales_out = None

    def compress(self, code=None):
        """code: a static dictionary from train_code() (then no histogram pass), or None."""
        if code is None:
            _check(lib().zc_compress_batch(self.arr, self.n, C.byref(self.p), _ptr(self.ws), self.ws.numel(), _stream()), "zc_compress_batch")
        else:
            _check(lib().zc_compress_batch_with_code(self.arr, self.n, C.byref(self.p), C.byref(code), _ptr(self.ws), self.ws.numel(), _stream()),
                   "zc_compress_batch_with_code")
        return [int(self.arr[i].out_bytes) for i in range(self.n)]

    def compress_async(self, code=None):
        """Queue the compression (with a static dictionary if one is given, else with codes built on the device)
        and return without waiting; call refresh_info() (which waits) before container(), decompress() or
        plan_decompress()."""
        if code is None:
            _check(lib().zc_compress_batch_async(self.arr, self.n, C.byref(self.p), _ptr(self.ws), self.ws.numel(), _stream()),
                   "zc_compress_batch_async")
        else:
            _check(lib().zc_compress_batch_with_code_async(self.arr, self.n, C.byref(self.p), C.byref(code), _ptr(self.ws), self.ws.numel(), _stream()),
                   "zc_compress_batch_with_code_async")

    def refresh_info(self):
        """Read every container's header back (blocking) after compress_async()."""
        for i in range(self.n):
            info = read_info(self.comp[i])
            self.arr[i].info = info
            self.arr[i].out_bytes = info.total_bytes
        return [int(self.arr[i].out_bytes) for i in range(self.n)]

    def container(self, i):
        return self.comp[i][:int(self.arr[i].out_bytes)]

    def prepare_outputs(self):
        dev = self.arena.device
        eb = elem_bits(self.p.format)
        self.out = [torch.empty(max((int(self.arr[i].n_elems) * eb + 7) // 8, 16), dtype=torch.uint8, device=dev) for i in range(self.n)]
        if scale_block(self.p.format):
            self.scales_out = [torch.empty(max(int(self.arr[i].n_elems) // scale_block(self.p.format), 16), dtype=torch.uint8, device=dev) for i in range(self.n)]
        for i in range(self.n):
            self.arr[i].d_dst = self.out[i].data_ptr()
            self.arr[i].d_scales_out = self.scales_out[i].data_ptr() if self.scales_out else None

    def set_outputs(self, outs, scales_out=None):
        """Decode into the caller's buffers (one uint8 CUDA tensor per tensor, each large enough) from the next plan on."""
        self.out, self.scales_out = list(outs), scales_out
        for i in range(self.n):
            self.arr[i].d_dst = self.out[i].data_ptr()
            self.arr[i].d_scales_out = scales_out[i].data_ptr() if scales_out else None

    def set_chunk_ids(self, ids):
        """ids: one int32 CUDA tensor of chunk ids per tensor (or None to decode whole tensors again).
        The next plan/decompress decodes only those chunks, densely, into fresh output buffers."""
        dev = self.arena.device
        self.ids = ids
        if ids is None:
            self.out = None
            for i in range(self.n):
                self.arr[i].d_chunk_ids = None
                self.arr[i].n_chunk_ids = 0
            return
        self.out = [torch.empty(max(ids[i].numel() * self.p.chunk_bytes, 16), dtype=torch.uint8, device=dev) for i in range(self.n)]
        for i in range(self.n):
            self.arr[i].d_chunk_ids = ids[i].data_ptr()
            self.arr[i].n_chunk_ids = ids[i].numel()
            self.arr[i].d_dst = self.out[i].data_ptr()

    def decompress(self):
        if self.out is None:
            self.prepare_outputs()
        _check(lib().zc_decompress_batch(self.arr, self.n, _ptr(self.ws), self.ws.numel(), _stream()), "zc_decompress_batch")
        return self.out

    def plan_decompress(self):
        """Queue the upload of descriptors and work lists on the current stream; returns the plan."""
        if self.out is None:
            self.prepare_outputs()
        self.plan = BatchPlan()
        _check(lib().zc_decompress_batch_plan(self.arr, self.n, _ptr(self.ws_plan), self.ws_plan.numel(), C.byref(self.plan), _stream()),
               "zc_decompress_batch_plan")
        return self.plan

    def run_decompress(self):
        """Enqueue the decode kernels on the plan left in the workspace by plan_decompress()."""
        _check(lib().zc_decompress_batch_run(C.byref(self.plan), _ptr(self.ws_plan), _stream()), "zc_decompress_batch_run")
        return self.out


def _types(*names):
    """Those of torch's types that this torch has (formats can be held as plain integers without them)."""
    return tuple(getattr(torch, name) for name in names if hasattr(torch, name))


_PAGE_TYPES = {FMT_BF16: _types("bfloat16", "int16", "uint16"), FMT_FP8_E4M3: _types("uint8", "int8", "float8_e4m3fn"),
               FMT_FP8_E5M2: _types("uint8", "int8", "float8_e5m2"), FMT_FP4_E2M1_MX: _types("uint8", "int8", "float4_e2m1fn_x2"),
               FMT_FP4_E2M1_NV: _types("uint8", "int8", "float4_e2m1fn_x2")}
_BLOCK_TYPES = {FMT_FP4_E2M1_MX: _types("uint8", "int8", "float8_e8m0fnu"), FMT_FP4_E2M1_NV: _types("uint8", "int8", "float8_e4m3fn")}
_ROW_TYPES = (torch.bfloat16, torch.int16, torch.uint16)


class PagedCache:
    """K and V of a batch of sequences in pages, as the attention and eviction calls take them.

    k_pages, v_pages: [n_pages, page_tokens, head_dim], contiguous, as stored (of the format's type, or as plain integers of
    its size; FP4: head_dim / 2 bytes, with k_blocks, v_blocks: [n_pages, page_tokens, head_dim / 32] (MX) or head_dim / 16 (NV), the
    block scales' bytes); table: int32 [n_seqs, n_heads, table_pages] of page numbers (one that is no page's: absent); lengths: int32
    [n_seqs], tokens in the cache; k_scales, v_scales: float32 [n_seqs, n_heads] or None.  The object holds the tensors
    and the descriptor; the lengths and the table are read on the device when a call runs, so they may change between calls."""

    def __init__(self, k_pages, v_pages, table, lengths, fmt, k_scales=None, v_scales=None, k_blocks=None, v_blocks=None):
        for name, t, dtype, dims in (("table", table, torch.int32, 3), ("lengths", lengths, torch.int32, 1)):
            if t.dtype != dtype or t.dim() != dims or not t.is_contiguous():
                raise ValueError("PagedCache: %s has to be a contiguous %s tensor of %d dimensions" % (name, dtype, dims))
        types = _PAGE_TYPES.get(fmt)
        if types is None:
            raise ZcError(ERR_UNSUPPORTED, "PagedCache")
        for t in (k_pages, v_pages):
            if t.dim() != 3 or t.dtype not in types or not t.is_contiguous() or t.shape != k_pages.shape:
                raise ValueError("PagedCache: pages have to be contiguous [n_pages, page_tokens, head_dim] tensors of the format's type")
        if lengths.shape[0] != table.shape[0]:
            raise ValueError("PagedCache: table and lengths are of different numbers of sequences")
        for t in (k_scales, v_scales):
            if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != tuple(table.shape[:2]) or not t.is_contiguous()):
                raise ValueError("PagedCache: scales have to be contiguous float32 [n_seqs, n_heads]")
        packed = 2 if fmt in _BLOCK_TYPES else 1                 # elements to an entry of the pages
        if packed == 2 and k_blocks is None and v_blocks is None:
            raise ZcError(ERR_UNSUPPORTED, "PagedCache: FP4 pages without block scales")
        for t in (k_blocks, v_blocks):
            if packed == 1 and t is not None:
                raise ValueError("PagedCache: the format has no block scales")
            if packed == 2 and (t is None or t.dtype not in _BLOCK_TYPES[fmt] or not t.is_contiguous() or
                                tuple(t.shape) != tuple(k_pages.shape[:2]) + (k_pages.shape[2] * 2 // scale_block(fmt),)):
                raise ValueError("PagedCache: block scales have to be contiguous [n_pages, page_tokens, head_dim / %d] bytes" % scale_block(fmt))
        self.device = k_pages.device
        if any(t is not None and t.device != self.device for t in (v_pages, table, lengths, k_scales, v_scales, k_blocks, v_blocks)):
            raise ValueError("PagedCache: tensors are on different devices")
        self.k_pages, self.v_pages, self.table, self.lengths = k_pages, v_pages, table, lengths
        self.k_scales, self.v_scales, self.k_blocks, self.v_blocks, self.fmt = k_scales, v_scales, k_blocks, v_blocks, fmt
        self.n_seqs, self.n_heads, self.table_pages = table.shape
        self.n_pages, self.page_tokens, self.head_dim = k_pages.shape[0], k_pages.shape[1], k_pages.shape[2] * packed
        self.capacity = self.table_pages * self.page_tokens
        c = self.c = KvCache()
        c.struct_size, c.format = C.sizeof(KvCache), fmt
        c.n_seqs, c.n_heads, c.head_dim, c.page_tokens = self.n_seqs, self.n_heads, self.head_dim, self.page_tokens
        c.table_pages, c.n_pages = self.table_pages, self.n_pages
        c.d_k_pages, c.d_v_pages, c.d_table, c.d_lengths = k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), lengths.data_ptr()
        c.d_k_scales = k_scales.data_ptr() if k_scales is not None else None
        c.d_v_scales = v_scales.data_ptr() if v_scales is not None else None
        c.d_k_block_scales = k_blocks.data_ptr() if k_blocks is not None else None
        c.d_v_block_scales = v_blocks.data_ptr() if v_blocks is not None else None
        self.ref = C.byref(c)


_MOST = 0xFFFFFFFF


def _check_numbers(what, **numbers):
    """The library takes 32 bits, and ctypes cuts what has more: -1 would be the largest number there is."""
    for name, x in numbers.items():
        if not 0 <= x <= _MOST:
            raise ValueError("%s: %s has to be in 0 .. 2^32 - 1, not %d" % (what, name, x))


def _least_in(a, m, lo, hi):
    """The least x >= 0 with lo <= a * x mod m <= hi (0 <= lo <= hi < m), or None.  Where no multiple of a is in the interval, a * x - m * y is in it for
    the least y for which m * y mod a is in the interval's negative: a smaller question of the same kind, as in Euclid's algorithm."""
    if lo == 0:
        return 0
    a %= m
    if a == 0:
        return None
    x = -(-lo // a)
    if a * x <= hi:
        return x
    y = _least_in(m % a, a, -hi % a, -lo % a)
    return None if y is None else -(-(lo + m * y) // a)


def _tokens_meet(off, n, a, b, dim):
    """Whether rows of dim elements at i * a and off + j * b (i, j < n; a, b >= dim) have elements in common."""
    if n == 1:
        return abs(off) < dim
    first, last = max(0, -((off + dim - 1) // b)), min(n - 1, ((n - 1) * a + dim - 1 - off) // b)      # the j whose rows reach what lies between the others' ends
    if first > last or a < 2 * dim:                              # (gaps of less than dim: no row fits)
        return first <= last
    lo = -(off + first * b + dim - 1) % a
    x = 0 if lo + 2 * dim - 2 >= a else _least_in(b, a, lo, lo + 2 * dim - 2)
    return x is not None and x <= last - first


def _rows_meet(k, v):
    """Whether rows of two BF16 tensors [n, heads, dim], none of which overlap among themselves, have elements in common."""
    (n, heads, dim), off = k.shape, (v.data_ptr() - k.data_ptr()) // 2
    strides = [t.stride()[:2] for t in (k, v)]
    reach = [a * (n - 1) + b * (heads - 1) + dim for a, b in strides]
    if not n or off >= reach[0] or -off >= reach[1]:
        return False
    levels = [(a, size) for a, b, size in zip(*strides, (n, heads)) if size > 1 and a == b]
    if len(levels) == (n > 1) + (heads > 1):                     # tokens and heads of one tensor: the differences next to 0 are among these
        near = [off]
        for stride, size in sorted(levels, reverse=True):
            near = [x + i * stride for x in near for i in (-(x // stride), -(x // stride) - 1) if -size < i < size]
        return any(abs(x) < dim for x in near)
    (a, a_head), (b, b_head) = strides
    return any(_tokens_meet(off + j * b_head - i * a_head, n, a, b, dim) for i in range(heads) for j in range(heads))


def _kv_rows(what, call, k, v, cache, q_start, results):
    """results: tensors of the caller's that are written to, 0 to 2 of (k, v)."""
    shape, heads, dim = k.shape, cache.n_heads, cache.head_dim
    n = shape[0] if len(shape) == 3 else 0
    for name, t in (("k", k), ("v", v)):
        if t.shape != (n, heads, dim) or t.stride(2) != 1 or t.dtype not in _ROW_TYPES:
            raise ValueError("%s: %s has to be [n_tokens, n_heads, head_dim] in BF16 with contiguous rows" % (what, name))
    for t in results:
        reach = dim                                              # elements from a row's first to the next free one
        for stride, size in sorted(zip(t.stride()[:2], shape)):
            if size > 1 and stride < reach:
                raise ValueError("%s: rows of %s overlap" % (what, "k" if t is k else "v"))
            reach += stride * (size - 1) if size > 1 else 0
    if len(results) == 2 and _rows_meet(k, v):
        raise ValueError("%s: rows of k and v overlap" % what)
    if (k.requires_grad or v.requires_grad) and torch.is_grad_enabled():
        raise ValueError("%s: there is no gradient through a stored cache: detach k and v, or call it under torch.no_grad()" % what)
    if q_start is None:
        if n != cache.n_seqs:
            raise ValueError("%s: without q_start there is one token per sequence" % what)
    elif q_start.dtype != torch.int32 or q_start.numel() != cache.n_seqs + 1 or not q_start.is_contiguous():
        raise ValueError("%s: q_start has to be contiguous int32 of n_seqs + 1 entries" % what)
    device, current = k.device, torch._C._cuda_getDevice() if k.is_cuda else -1       # (the kernels go to the current GPU's stream)
    if device.index != current or cache.device != device or v.device != device or (q_start is not None and q_start.device != device):
        raise ValueError("%s: tensors have to be on one GPU, the current one" % what)
    (kt, kh, _), (vt, vh, _) = k.stride(), v.stride()
    if n == 1 or heads == 1:                                     # the stride of a dimension of one element is any number
        kt, vt = (0, 0) if n == 1 else (kt, vt)
        kh, vh = (0, 0) if heads == 1 else (kh, vh)
    a = KvRows.from_buffer_copy(_pack_kv_rows(_KV_ROWS_BYTES, n, k.data_ptr(), v.data_ptr(), kt, kh, vt, vh, 0 if q_start is None else q_start.data_ptr()))
    st = call(C.byref(a), cache.ref, torch._C._cuda_getCurrentRawStream(current))
    if st != OK:
        raise ZcError(st, what)


def write_kv(k, v, cache, q_start=None):
    """Quantises BF16 keys and values [n_tokens, n_heads, head_dim] into the pages of a PagedCache: what the last tokens of every
    sequence are, whose lengths count them already (as attend() takes its queries, so that a step is: lengths += 1, write_kv, attend).

    q_start: int32 [n_seqs + 1], where each sequence's tokens begin (None: one token per sequence).  FP8: divided by the cache's
    scales, the largest number where they are beyond it; FP4: with a scale for every block, which is written to k_blocks and v_blocks."""
    _kv_rows("zc_kv_write", lib().zc_kv_write, k, v, cache, q_start, ())


def read_kv(cache, q_start=None, n_tokens=None, k=None, v=None):
    """The last tokens of every sequence of a PagedCache as attention sees them: (k, v), BF16 [n_tokens, n_heads, head_dim].

    q_start: int32 [n_seqs + 1], where each sequence's tokens begin (None: one token, the last, per sequence); n_tokens: rows of the
    results (needed with q_start unless k or v is given; rows of tokens of no sequence are left as they are); k, v: where the results go."""
    if n_tokens is None:
        n_tokens = k.shape[0] if k is not None else v.shape[0] if v is not None else cache.n_seqs
        if k is None and v is None and q_start is not None:
            raise ValueError("zc_kv_read: with q_start, n_tokens says how many rows there are")
    _check_numbers("zc_kv_read", n_tokens=n_tokens)
    results = [t for t in (k, v) if t is not None]
    size = (n_tokens, cache.n_heads, cache.head_dim)
    if k is None:
        k = cache.k_pages.new_empty(size, dtype=torch.bfloat16)
        if v is None:
            v = torch.empty_like(k)
    elif k.shape[0] != n_tokens:
        raise ValueError("zc_kv_read: k has to be [n_tokens, n_heads, head_dim] in BF16 with contiguous rows")
    if v is None:
        v = cache.k_pages.new_empty(size, dtype=torch.bfloat16)
    _kv_rows("zc_kv_read", lib().zc_kv_read, k, v, cache, q_start, results)
    return k, v


def _attend(what, q, prefix, cache, q_start, max_q_len, window, sinks, scale, max_kv_len, max_prefix_len, out, lse, weights, weights_out, ws):
    if q.dim() != 3 or q.shape[2] != cache.head_dim or q.stride(2) != 1 or q.dtype not in _ROW_TYPES:
        raise ValueError("%s: q has to be [n_tokens, n_q_heads, head_dim] in BF16 with contiguous rows" % what)
    n, heads, dim = q.shape
    if out is None:
        out = q.new_empty((n, heads, dim))
    elif out.shape != q.shape or out.stride(2) != 1 or out.dtype not in _ROW_TYPES:
        raise ValueError("%s: out has to have q's shape and type, with contiguous rows" % what)
    elif (n > 1 and out.stride(0) < dim) or (heads > 1 and out.stride(1) < dim):
        raise ValueError("%s: rows of out overlap" % what)
    if lse is None:
        lse = q.new_empty((n, heads), dtype=torch.float32)
    elif lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous():
        raise ValueError("%s: lse has to be contiguous float32 [n_tokens, n_q_heads]" % what)
    if q_start is not None and (q_start.dtype != torch.int32 or q_start.numel() != cache.n_seqs + 1 or not q_start.is_contiguous()):
        raise ValueError("%s: q_start has to be contiguous int32 of n_seqs + 1 entries" % what)
    for t in (weights, weights_out):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (cache.n_seqs, cache.n_heads, cache.capacity) or not t.is_contiguous()):
            raise ValueError("%s: weights have to be contiguous float32 [n_seqs, n_heads, table_pages * page_tokens]" % what)
    if ws is not None and not ws.is_contiguous():
        raise ValueError("%s: ws has to be contiguous" % what)
    if max_q_len is None:
        max_q_len = 1 if q_start is None else max(n, 1)
    if not (0 <= max_q_len <= _MOST and 0 <= window <= _MOST and 0 <= sinks <= _MOST and 0 <= max_kv_len <= _MOST and 0 <= max_prefix_len <= _MOST):
        _check_numbers(what, max_q_len=max_q_len, window=window, sinks=sinks, max_kv_len=max_kv_len, max_prefix_len=max_prefix_len)
    if (q.requires_grad or (weights is not None and weights.requires_grad)) and torch.is_grad_enabled():
        raise ValueError("%s: there is no gradient through a stored cache: detach q and weights, or call it under torch.no_grad()" % what)
    device, current = q.device, torch._C._cuda_getDevice() if q.is_cuda else -1       # (the kernels go to the current GPU's stream)
    if device.index != current or cache.device != device or out.device != device or lse.device != device or \
            any(t is not None and t.device != device for t in (q_start, weights, weights_out, ws, prefix)):
        raise ValueError("%s: tensors have to be on one GPU, the current one" % what)
    strides = q.stride()[:2] + out.stride()[:2]
    if n == 1 or heads == 1:                                     # the stride of a dimension of one element is any number
        strides = [0 if size == 1 else stride for size, stride in zip((n, heads, n, heads), strides)]
    a = AttendArgs.from_buffer_copy(_pack_attend_args(
        _ATTEND_ARGS_BYTES, n, heads, max_q_len, window, sinks, max_kv_len, max_prefix_len, dim ** -0.5 if scale is None else C.c_float(scale).value, 0,
        q.data_ptr(), out.data_ptr(), *strides, 0 if q_start is None else q_start.data_ptr(), lse.data_ptr(),
        0 if weights is None else weights.data_ptr(), 0 if weights_out is None else weights_out.data_ptr()))
    L, ref = lib(), C.byref(a)
    at, size = (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())
    if ws is None:
        size = L.zc_attend_workspace_bytes(ref, None if prefix is None else prefix.ref, cache.ref)
        if size:
            ws = torch.empty(size, dtype=torch.uint8, device=q.device)
            at = ws.data_ptr()
    stream = torch._C._cuda_getCurrentRawStream(current)
    st = L.zc_attend(ref, cache.ref, at, size, stream) if prefix is None else L.zc_attend_shared(ref, prefix.ref, cache.ref, at, size, stream)
    if st != OK:
        raise ZcError(st, what)
    return out, lse


def attend(q, cache, q_start=None, max_q_len=None, window=0, sinks=0, scale=None, max_kv_len=0, out=None, lse=None, weights=None, weights_out=None, ws=None):
    """Attention of BF16 queries [n_tokens, n_q_heads, head_dim] over a PagedCache; returns (out, lse).

    q_start: int32 [n_seqs + 1], where each sequence's query tokens begin (None: one token per sequence).  max_q_len: no sequence
    has more of them (None: any number); kernels are chosen by it, so it is worth giving where all sequences go on by a token or a
    few, and those that bring a prompt are best given a call of their own.  window: how many of the latest tokens a query sees,
    itself included (0: all); sinks: how many of the first ones it always sees.  scale: of the logits (None: head_dim ** -0.5).
    max_kv_len: no length is above it (0: the table's room).  weights_out: also leaves weights (None: zeros) plus the attention
    weight given to each token there."""
    return _attend("zc_attend", q, None, cache, q_start, max_q_len, window, sinks, scale, max_kv_len, 0, out, lse, weights, weights_out, ws)


def attend_shared(q, prefix, cache, q_start=None, max_q_len=None, window=0, sinks=0, scale=None, max_kv_len=0, max_prefix_len=0, out=None, lse=None, ws=None):
    """attend() for sequences whose first tokens are those of `prefix` (a PagedCache of one sequence), read once for all of
    them; `cache` holds what follows in each."""
    return _attend("zc_attend_shared", q, prefix, cache, q_start, max_q_len, window, sinks, scale, max_kv_len, max_prefix_len, out, lse, None, None, ws)


def evict(cache, weights, keep, into, into_weights=None, sinks=0, recent=0, kept=None):
    """Leaves `keep` tokens per sequence and head: the first `sinks`, the last `recent`, and of the others those with the largest
    weights (float32 [n_seqs, n_heads, table_pages * page_tokens]); they go to the pages of `into` (another PagedCache),
    whose lengths are set.  Returns their numbers, int32 [n_seqs, n_heads, keep], ascending, -1 behind the last."""
    _check_numbers("zc_evict", keep=keep, sinks=sinks, recent=recent)
    if kept is None:
        kept = torch.empty((cache.n_seqs, cache.n_heads, keep), dtype=torch.int32, device=weights.device)
    elif kept.dtype != torch.int32 or tuple(kept.shape) != (cache.n_seqs, cache.n_heads, keep) or not kept.is_contiguous():
        raise ValueError("zc_evict: kept has to be contiguous int32 [n_seqs, n_heads, keep]")
    for t, c in ((weights, cache), (into_weights, into)):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (c.n_seqs, c.n_heads, c.capacity) or not t.is_contiguous()):
            raise ValueError("zc_evict: weights have to be contiguous float32 [n_seqs, n_heads, table_pages * page_tokens]")
    if into_weights is not None and weights.requires_grad and torch.is_grad_enabled():
        raise ValueError("zc_evict: no gradient goes to into_weights: detach weights, or call it under torch.no_grad()")
    if not weights.is_cuda or weights.device.index != torch._C._cuda_getDevice() or any(t is not None and t.device != weights.device for t in (cache, into, into_weights, kept)):
        raise ValueError("zc_evict: tensors have to be on one GPU, the current one")
    st = lib().zc_evict(cache.ref, weights.data_ptr(), keep, sinks, recent, into.ref, into_weights.data_ptr() if into_weights is not None else None,
                        kept.data_ptr(), _stream())
    _check(st, "zc_evict")
    return kept
