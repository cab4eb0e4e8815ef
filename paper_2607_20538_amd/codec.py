"""ctypes binding of the codec library's C ABI (include/codec_gauge.h).

Argument marshalling only: every step of the codec runs in the HIP library.  Functions
carry the C names (gauge_make, kv_encode, kv_decode, kv_append_step, cache_bytes,
gauge_device_bytes) and accept torch tensors for device buffers; the stream defaults to
torch's current stream.  A missing library raises instead of falling back to anything.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcodecgauge.so")

CG_OK, CG_ERR_ARG, CG_ERR_SHAPE, CG_ERR_ALIGN, CG_ERR_UNSUPPORTED, CG_ERR_NOT_ORTHOGONAL, CG_ERR_CAPACITY, \
    CG_ERR_DEVICE = range(8)
CG_FLAG_NONFINITE, CG_FLAG_SIDE_OVERFLOW, CG_FLAG_POS_RANGE, CG_FLAG_POOL_EMPTY = 1, 2, 4, 8
GAUGE_IDENTITY, GAUGE_HAAR, GAUGE_DCT2, GAUGE_HADAMARD, GAUGE_EXPM, GAUGE_USER = range(6)
PASSTHROUGH, BLOCK_UNIFORM, KIVI, ZFP = 0, 1, 2, 3
DTYPE_BF16, DTYPE_F32 = 0, 1
ROPE_HALF, ROPE_PAIRS = 0, 1
ROPE_NONE, ROPE_LINEAR, ROPE_RAMP = 0, 1, 2
TREE_MOST = 1024  # nodes of a row's trees

EXPORTS = ["cg_status_str", "gauge_device_bytes", "gauge_make", "cache_bytes", "kv_encode", "kv_decode",
           "kv_append_step", "spectral_workspace_bytes", "kv_spectral_stats", "gauge_grad_workspace_bytes",
           "kv_gauge_grad", "attend_workspace_bytes", "kv_attend",
           "kv_attend_noalloc",
           "attend_paged_workspace_bytes", "kv_attend_paged", "kv_encode_paged", "kv_append_paged",
           "kv_page_map", "kv_page_release", "rope_make", "kv_rope", "kv_append_slots",
           "attend_chunk_workspace_bytes", "attend_chunk_workspace_limit", "kv_attend_chunk_paged",
           "kv_page_trim", "kv_tree_map", "kv_tree_map_window", "kv_append_rope", "attend_tree_workspace_bytes", "kv_attend_tree_paged",
           "kv_tree_accept", "kv_tree_keep", "cg_selftest", "cg_stream_probe"]


class GaugeShape(C.Structure):
    _fields_ = [("L", C.c_int32), ("H", C.c_int32), ("d", C.c_int32), ("g", C.c_int32)]


class PageTable(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("max_pages", C.c_int32), ("page_size", C.c_int32)]


class PagePoolStruct(C.Structure):
    _fields_ = [("free_pages", C.c_void_p), ("free_count", C.c_void_p), ("n_pages", C.c_int32)]


class Rope(C.Structure):
    _fields_ = [("d_rot", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32), ("train_len", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("amplitude", C.c_double)]


class RopePlan(C.Structure):
    _fields_ = [("d_rot", C.c_int32), ("layout", C.c_int32), ("amplitude", C.c_float), ("reserved", C.c_int32),
                ("step", C.c_uint64 * 128)]


class CodecStruct(C.Structure):
    _fields_ = [("backend", C.c_int32), ("bits", C.c_int32), ("block_c", C.c_int32), ("key_tokens", C.c_int32),
                ("val_channels", C.c_int32), ("residual", C.c_int32), ("block_t", C.c_int32)]


class KvView(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32), ("L", C.c_int32), ("B", C.c_int32), ("H", C.c_int32),
                ("T", C.c_int32), ("d", C.c_int32), ("stride_l", C.c_int64), ("stride_b", C.c_int64),
                ("stride_h", C.c_int64), ("stride_t", C.c_int64)]


class CacheStruct(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("side", C.c_void_p), ("residual", C.c_void_p), ("L", C.c_int32),
                ("B", C.c_int32), ("H", C.c_int32), ("T_cap", C.c_int32), ("d", C.c_int32), ("len", C.c_int32)]


class CodecError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn}: {status_str(status)} (status {status})")
        self.status = status


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run paper_2607_20538_amd/build.py")
        L = C.CDLL(LIB_PATH)
        p, i32, u64 = C.c_void_p, C.c_int32, C.c_uint64
        L.cg_status_str.argtypes = [i32]
        L.cg_status_str.restype = C.c_char_p
        L.gauge_device_bytes.argtypes = [GaugeShape]
        L.gauge_device_bytes.restype = C.c_size_t
        L.gauge_make.argtypes = [i32, GaugeShape, u64, p, p, p, p]
        L.gauge_make.restype = i32
        L.cache_bytes.argtypes = [C.POINTER(CodecStruct), i32, i32, i32, i32, i32, i32, p, p, p]
        L.cache_bytes.restype = i32
        L.kv_encode.argtypes = [i32, C.POINTER(KvView), p, GaugeShape, C.POINTER(CodecStruct),
                                C.POINTER(CacheStruct), i32, p, p]
        L.kv_encode.restype = i32
        L.kv_decode.argtypes = [i32, C.POINTER(CacheStruct), p, GaugeShape, C.POINTER(CodecStruct), p, i32,
                                C.POINTER(KvView), p, p]
        L.kv_decode.restype = i32
        L.kv_append_step.argtypes = [i32, i32, C.POINTER(KvView), C.POINTER(KvView), p, p, GaugeShape,
                                     C.POINTER(CodecStruct), C.POINTER(CacheStruct), C.POINTER(CacheStruct),
                                     C.POINTER(KvView), C.POINTER(KvView), p, p]
        L.kv_append_step.restype = i32
        L.spectral_workspace_bytes.argtypes = [GaugeShape, i32]
        L.spectral_workspace_bytes.restype = C.c_size_t
        L.kv_spectral_stats.argtypes = [i32, C.POINTER(KvView), p, GaugeShape, i32, C.c_float, p, p, p, p]
        L.kv_spectral_stats.restype = i32
        L.gauge_grad_workspace_bytes.argtypes = [GaugeShape, i32, i32, i32]
        L.gauge_grad_workspace_bytes.restype = C.c_size_t
        L.kv_gauge_grad.argtypes = [i32, C.POINTER(KvView), p, p, GaugeShape, i32, C.c_float, C.c_float, C.c_float, p,
                                    p, p, p]
        L.kv_gauge_grad.restype = i32
        L.attend_workspace_bytes.argtypes = [GaugeShape, i32, i32, i32, i32]
        L.attend_workspace_bytes.restype = C.c_size_t
        L.kv_attend.argtypes = [i32, i32, C.POINTER(KvView), C.POINTER(CacheStruct), C.POINTER(CacheStruct), p,
                                GaugeShape, C.POINTER(CodecStruct), p, C.c_float, C.POINTER(KvView), p, p, p]
        L.kv_attend.restype = i32
        L.kv_attend_noalloc.argtypes = [i32, i32, C.POINTER(KvView), C.POINTER(CacheStruct), C.POINTER(CacheStruct),
                                        p, GaugeShape, C.POINTER(CodecStruct), p, C.c_float, C.POINTER(KvView), p, p]
        L.kv_attend_noalloc.restype = i32
        L.attend_paged_workspace_bytes.argtypes = [GaugeShape, i32, i32, i32, i32, i32]
        L.attend_paged_workspace_bytes.restype = C.c_size_t
        L.kv_attend_paged.argtypes = [i32, i32, C.POINTER(KvView), C.POINTER(CacheStruct), C.POINTER(CacheStruct),
                                      C.POINTER(PageTable), p, GaugeShape, C.POINTER(CodecStruct), p, C.c_float,
                                      C.POINTER(KvView), p, p, p]
        L.kv_attend_paged.restype = i32
        L.kv_encode_paged.argtypes = [i32, C.POINTER(KvView), C.POINTER(PageTable), p, GaugeShape,
                                      C.POINTER(CodecStruct), C.POINTER(CacheStruct), i32, p, p]
        L.kv_encode_paged.restype = i32
        L.kv_append_paged.argtypes = [i32, i32, C.POINTER(KvView), C.POINTER(KvView), p, C.POINTER(PageTable), p,
                                      GaugeShape, C.POINTER(CodecStruct), C.POINTER(CacheStruct),
                                      C.POINTER(CacheStruct), p, p]
        L.kv_append_paged.restype = i32
        L.kv_page_map.argtypes = [p, p, i32, C.POINTER(PagePoolStruct), p, i32, i32, i32, p, p, p, p, p, p]
        L.kv_page_map.restype = i32
        L.kv_page_release.argtypes = [p, p, i32, C.POINTER(PagePoolStruct), p, i32, i32, p, p]
        L.kv_page_release.restype = i32
        L.rope_make.argtypes = [C.POINTER(Rope), C.POINTER(RopePlan)]
        L.rope_make.restype = i32
        L.kv_rope.argtypes = [C.POINTER(RopePlan), C.POINTER(KvView), C.POINTER(KvView), C.POINTER(KvView),
                              C.POINTER(KvView), p, i32, p]
        L.kv_rope.restype = i32
        L.kv_append_slots.argtypes = [i32, i32, C.POINTER(KvView), C.POINTER(KvView), p, p, GaugeShape,
                                      C.POINTER(CodecStruct), C.POINTER(CacheStruct), C.POINTER(CacheStruct), p, p]
        L.kv_append_slots.restype = i32
        L.attend_chunk_workspace_bytes.argtypes = [GaugeShape] + [i32] * 9
        L.attend_chunk_workspace_bytes.restype = C.c_size_t
        L.attend_chunk_workspace_limit.argtypes = [GaugeShape] + [i32] * 6
        L.attend_chunk_workspace_limit.restype = C.c_size_t
        L.kv_attend_chunk_paged.argtypes = [i32, i32, C.POINTER(KvView), p, i32, i32, C.POINTER(CacheStruct),
                                            C.POINTER(CacheStruct), C.POINTER(PageTable), p, GaugeShape,
                                            C.POINTER(CodecStruct), p, C.c_float, i32, i32, C.POINTER(KvView), p, p, p]
        L.kv_attend_chunk_paged.restype = i32
        L.kv_page_trim.argtypes = L.kv_page_release.argtypes
        L.kv_page_trim.restype = i32
        L.kv_tree_map.argtypes = [p, p, p, i32, i32, i32, p, p, p, p]
        L.kv_tree_map.restype = i32
        L.kv_tree_map_window.argtypes = [p, p, p, i32, i32, i32, i32, i32, p, p, p, p]
        L.kv_tree_map_window.restype = i32
        L.kv_append_rope.argtypes = [i32, i32, C.POINTER(RopePlan), C.POINTER(KvView), C.POINTER(KvView),
                                     C.POINTER(KvView), C.POINTER(KvView), p, p, p, GaugeShape, C.POINTER(CodecStruct),
                                     C.POINTER(CacheStruct), C.POINTER(CacheStruct), p, p]
        L.kv_append_rope.restype = i32
        L.attend_tree_workspace_bytes.argtypes = [GaugeShape] + [i32] * 6
        L.attend_tree_workspace_bytes.restype = C.c_size_t
        L.kv_attend_tree_paged.argtypes = [i32, i32, C.POINTER(KvView), p, i32, i32, p, i32, p, C.POINTER(CacheStruct),
                                           C.POINTER(CacheStruct), C.POINTER(PageTable), p, GaugeShape,
                                           C.POINTER(CodecStruct), p, C.c_float, i32, i32, C.POINTER(KvView), p, p, p]
        L.kv_attend_tree_paged.restype = i32
        L.kv_tree_accept.argtypes = [p, p, p, p, p, i32, i32, p, p, p, p, p]
        L.kv_tree_accept.restype = i32
        L.kv_tree_keep.argtypes = [i32, i32, p, p, p, p, i32, i32, C.POINTER(PageTable), GaugeShape,
                                   C.POINTER(CodecStruct), C.POINTER(CacheStruct), C.POINTER(CacheStruct), p, p, p]
        L.kv_tree_keep.restype = i32
        L.cg_selftest.argtypes = [i32, p, p]
        L.cg_selftest.restype = i32
        L.cg_stream_probe.argtypes = [p, C.c_int64, p, C.c_int64, p]
        L.cg_stream_probe.restype = i32
        _lib = L
    return _lib


def status_str(status: int) -> str:
    return lib().cg_status_str(int(status)).decode()


def _check(fn: str, rc: int):
    if rc != CG_OK:
        raise CodecError(fn, rc)


@dataclasses.dataclass(frozen=True)
class Codec:
    backend: int = BLOCK_UNIFORM
    bits: int = 4
    block_c: int = 64
    key_tokens: int = 32
    val_channels: int = 64
    residual: int = 128
    block_t: int = 1

    def struct(self) -> CodecStruct:
        return CodecStruct(self.backend, self.bits, self.block_c, self.key_tokens, self.val_channels, self.residual,
                           self.block_t)


def shape(L: int, H: int, d: int, g: int) -> GaugeShape:
    return GaugeShape(L, H, d, g)


def _ptr(t) -> int | None:
    if t is None:
        return None
    return t.data_ptr()


_raw_stream = None


def _stream(stream) -> int | None:
    """The stream handle to launch on: the caller's, else torch's current stream of its current
    device.  Once torch has initialised the device, the handle is asked for directly; building
    torch's Stream object (and asking for the device count) took 3.6 of a call's 9.8 us."""
    global _raw_stream
    if stream is not None:
        return int(stream)
    import torch

    if _raw_stream is None:
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", False)
    if _raw_stream and torch.cuda.is_initialized():
        return _raw_stream(torch.cuda.current_device())
    if torch.cuda.is_available():
        return torch.cuda.current_stream().cuda_stream
    return None


_dtypes = None


def view(t) -> KvView:
    """cg_kv_view of a torch tensor [L][B][H][T][d] (bf16 or float32, channel stride 1)."""
    global _dtypes
    if _dtypes is None:
        import torch

        _dtypes = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}
    s = t.stride()
    if len(s) != 5 or s[4] != 1:
        raise ValueError("KV view needs a [L][B][H][T][d] tensor with unit channel stride")
    return KvView(t.data_ptr(), _dtypes[t.dtype], *t.shape, *s[:4])


# ------------------------------------------------------------------------------------------
# entry points
# ------------------------------------------------------------------------------------------

def gauge_device_bytes(shp: GaugeShape) -> int:
    return int(lib().gauge_device_bytes(shp))


def gauge_make(kind: int, shp: GaugeShape, seed: int = 0, params: np.ndarray | None = None, G_host=True,
               G_dev=None, stream=None):
    """Returns (G_host float32 [L][2][H][R][g][g] or None, G_dev)."""
    R = shp.d // shp.g
    host = np.zeros((shp.L, 2, shp.H, R, shp.g, shp.g), dtype=np.float32) if G_host is True else G_host
    par = None if params is None else np.ascontiguousarray(params, dtype=np.float32)
    rc = lib().gauge_make(kind, shp, seed, None if par is None else par.ctypes.data,
                          None if host is None else host.ctypes.data, _ptr(G_dev), _stream(stream))
    _check("gauge_make", rc)
    return host, G_dev


def alloc_gauge(shp: GaugeShape, device="cuda"):
    import torch

    return torch.empty(gauge_device_bytes(shp), dtype=torch.uint8, device=device)


def cache_bytes(codec: Codec, s: int, L: int, B: int, H: int, T_cap: int, d: int):
    c, sd, r = C.c_size_t(), C.c_size_t(), C.c_size_t()
    cs = codec.struct()
    rc = lib().cache_bytes(C.byref(cs), s, L, B, H, T_cap, d, C.addressof(c), C.addressof(sd), C.addressof(r))
    _check("cache_bytes", rc)
    return c.value, sd.value, r.value


class Cache:
    """Device buffers of one compressed K or V cache (flat uint8 tensors)."""

    def __init__(self, codec: Codec, s: int, L: int, B: int, H: int, T_cap: int, d: int, device="cuda"):
        import torch

        nc, ns, nr = cache_bytes(codec, s, L, B, H, T_cap, d)
        mk = lambda n: torch.zeros(max(n, 16), dtype=torch.uint8, device=device) if n else None
        self.codes, self.side, self.residual = mk(nc), mk(ns), mk(nr)
        self.nbytes = (nc, ns, nr)
        self.L, self.B, self.H, self.T_cap, self.d = L, B, H, T_cap, d
        self.len = 0

    def struct(self) -> CacheStruct:
        return CacheStruct(_ptr(self.codes), _ptr(self.side), _ptr(self.residual), self.L, self.B, self.H,
                           self.T_cap, self.d, self.len)


def kv_encode(s: int, X, G_dev, shp: GaugeShape, codec: Codec, cache: Cache, t0: int = 0, err_flag=None,
              stream=None):
    v, cs, ks = view(X), codec.struct(), cache.struct()
    rc = lib().kv_encode(s, C.byref(v), _ptr(G_dev), shp, C.byref(cs), C.byref(ks), t0, _ptr(err_flag),
                         _stream(stream))
    _check("kv_encode", rc)


def kv_decode(s: int, cache: Cache, G_dev, shp: GaugeShape, codec: Codec, t0: int, Xhat, err_flag=None,
              stream=None, lens=None):
    """lens: optional device int32 tensor [B] of per-row lengths (else every row holds cache.len)."""
    v, cs, ks = view(Xhat), codec.struct(), cache.struct()
    rc = lib().kv_decode(s, C.byref(ks), _ptr(G_dev), shp, C.byref(cs), _ptr(lens), t0, C.byref(v),
                         _ptr(err_flag), _stream(stream))
    _check("kv_decode", rc)


def cg_selftest(which: int, mismatches_dev, stream=None):
    """Adds the mismatch count of device self-test `which` to the uint64 device tensor."""
    rc = lib().cg_selftest(which, _ptr(mismatches_dev), _stream(stream))
    _check("cg_selftest", rc)


def cg_stream_probe(src, read_bytes: int, dst, write_bytes: int, stream=None):
    """Streams `read_bytes` of device tensor `src` and writes `write_bytes` into `dst` in one
    kernel (the HBM ceiling of that read / write mix; `dst` is left unspecified)."""
    if src.nbytes < read_bytes or (write_bytes and dst.nbytes < write_bytes):
        raise ValueError("cg_stream_probe: buffer smaller than the byte count")
    rc = lib().cg_stream_probe(_ptr(src), read_bytes, _ptr(dst), write_bytes, _stream(stream))
    _check("cg_stream_probe", rc)


def kv_append_step(l0: int, l1: int, k_new, v_new, pos, G_dev, shp: GaugeShape, codec: Codec, kc: Cache,
                   vc: Cache, k_hist=None, v_hist=None, err_flag=None, stream=None):
    kn, vn, cs, kcs, vcs = view(k_new), view(v_new), codec.struct(), kc.struct(), vc.struct()
    kh = None if k_hist is None else C.byref(view(k_hist))
    vh = None if v_hist is None else C.byref(view(v_hist))
    rc = lib().kv_append_step(l0, l1, C.byref(kn), C.byref(vn), _ptr(pos), _ptr(G_dev), shp, C.byref(cs),
                              C.byref(kcs), C.byref(vcs), kh, vh, _ptr(err_flag), _stream(stream))
    _check("kv_append_step", rc)


def spectral_workspace_bytes(shp: GaugeShape, block_t: int) -> int:
    return int(lib().spectral_workspace_bytes(shp, block_t))


def kv_spectral_stats(s: int, X, G_dev, shp: GaugeShape, block_t: int, tau: float, workspace, stats, energy=None,
                      stream=None):
    """Spectral statistics of G X (section 4.2) into the device float64 tensors stats [L][4] and,
    if given, energy [L][block_t][d]; workspace: device buffer of spectral_workspace_bytes."""
    v = view(X)
    rc = lib().kv_spectral_stats(s, C.byref(v), _ptr(G_dev), shp, block_t, tau, _ptr(workspace), _ptr(stats),
                                 _ptr(energy), _stream(stream))
    _check("kv_spectral_stats", rc)


def gauge_grad_workspace_bytes(shp: GaugeShape, B: int, T: int, block_t: int) -> int:
    return int(lib().gauge_grad_workspace_bytes(shp, B, T, block_t))


def kv_gauge_grad(s: int, X, A, G_dev, shp: GaugeShape, block_t: int, tau: float, lambda_f: float, lambda_r: float,
                  workspace, stats, grad, stream=None):
    """Gradient of the training objective (section 4.2) with respect to the generators A (device
    float32 [L][2][H][R][g][g], G = exp(A - A^T)) into the device float64 tensors grad
    [L][H][R][g][g] and stats [L][4]; workspace: device buffer of gauge_grad_workspace_bytes."""
    v = view(X)
    rc = lib().kv_gauge_grad(s, C.byref(v), _ptr(A), _ptr(G_dev), shp, block_t, tau, lambda_f, lambda_r,
                             _ptr(workspace), _ptr(stats), _ptr(grad), _stream(stream))
    _check("kv_gauge_grad", rc)


def attend_workspace_bytes(shp: GaugeShape, nl: int, B: int, Hq: int, T_cap: int) -> int:
    return int(lib().attend_workspace_bytes(shp, nl, B, Hq, T_cap))


def kv_attend(l0: int, l1: int, q, kc: Cache, vc: Cache, G_dev, shp: GaugeShape, codec: Codec, lens, scale: float,
              out, workspace=None, err_flag=None, stream=None):
    """Decode-phase attention of q [l1-l0][B][Hq][1][d] over the compressed caches into out (same
    shape); lens: device int32 [B] positions per row, or None for the caches' len."""
    qv, ov, cs, kcs, vcs = view(q), view(out), codec.struct(), kc.struct(), vc.struct()
    rc = lib().kv_attend(l0, l1, C.byref(qv), C.byref(kcs), C.byref(vcs), _ptr(G_dev), shp, C.byref(cs), _ptr(lens),
                         float(scale), C.byref(ov), _ptr(workspace), _ptr(err_flag), _stream(stream))
    _check("kv_attend", rc)


def kv_attend_noalloc(l0: int, l1: int, q, kc: Cache, vc: Cache, G_dev, shp: GaugeShape, codec: Codec, lens,
                      scale: float, out, err_flag=None, stream=None):
    """kv_attend without a workspace: split rows' partials go to the library's device scratch."""
    qv, ov, cs, kcs, vcs = view(q), view(out), codec.struct(), kc.struct(), vc.struct()
    rc = lib().kv_attend_noalloc(l0, l1, C.byref(qv), C.byref(kcs), C.byref(vcs), _ptr(G_dev), shp, C.byref(cs),
                                 _ptr(lens), float(scale), C.byref(ov), _ptr(err_flag), _stream(stream))
    _check("kv_attend_noalloc", rc)


def page_table(pages, page_size: int) -> PageTable:
    """cg_page_table of a contiguous device int32 tensor pages [B][max_pages] (columns cut from a wider table are
    not one: their rows lie further apart)."""
    if pages.dim() != 2:
        raise ValueError("page_table: pages must be [B][max_pages]")
    _int32("page_table", None, pages=pages)
    pt = PageTable(_ptr(pages), int(pages.shape[1]), int(page_size))
    pt.tensor = pages  # lives as long as the table
    return pt


def attend_paged_workspace_bytes(shp: GaugeShape, nl: int, B: int, Hq: int, max_pages: int, page_size: int) -> int:
    return int(lib().attend_paged_workspace_bytes(shp, nl, B, Hq, max_pages, page_size))


def kv_attend_paged(l0: int, l1: int, q, kc: Cache, vc: Cache, pt: PageTable, G_dev, shp: GaugeShape, codec: Codec,
                    lens, scale: float, out, workspace=None, err_flag=None, stream=None):
    """kv_attend over page pools kc / vc (their B counts pages, T_cap = page size) through pt."""
    qv, ov, cs, kcs, vcs = view(q), view(out), codec.struct(), kc.struct(), vc.struct()
    rc = lib().kv_attend_paged(l0, l1, C.byref(qv), C.byref(kcs), C.byref(vcs), C.byref(pt), _ptr(G_dev), shp,
                               C.byref(cs), _ptr(lens), float(scale), C.byref(ov), _ptr(workspace), _ptr(err_flag),
                               _stream(stream))
    _check("kv_attend_paged", rc)


def kv_encode_paged(s: int, X, pt: PageTable, G_dev, shp: GaugeShape, codec: Codec, cache: Cache, t0: int = 0,
                    err_flag=None, stream=None):
    v, cs, ks = view(X), codec.struct(), cache.struct()
    rc = lib().kv_encode_paged(s, C.byref(v), C.byref(pt), _ptr(G_dev), shp, C.byref(cs), C.byref(ks), t0,
                               _ptr(err_flag), _stream(stream))
    _check("kv_encode_paged", rc)


def kv_append_paged(l0: int, l1: int, k_new, v_new, pos, pt: PageTable, G_dev, shp: GaugeShape, codec: Codec,
                    kc: Cache, vc: Cache, err_flag=None, stream=None):
    kn, vn, cs, kcs, vcs = view(k_new), view(v_new), codec.struct(), kc.struct(), vc.struct()
    rc = lib().kv_append_paged(l0, l1, C.byref(kn), C.byref(vn), _ptr(pos), C.byref(pt), _ptr(G_dev), shp,
                               C.byref(cs), C.byref(kcs), C.byref(vcs), _ptr(err_flag), _stream(stream))
    _check("kv_append_paged", rc)


# ------------------------------------------------------------------------------------------
# a serving step over paged caches: tables and slots, rotary positions, packed tokens
# ------------------------------------------------------------------------------------------

_int32_type = _current = None


def _on_device(fn: str, **tensors):
    """The named tensors lie on the device that is current (the library launches there).  None is left out.
    (Five tensors took 1.0 of a call's 10 us with torch's own question for the device and an import in here.)"""
    global _current
    if _current is None:
        import torch

        _current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    dev = -1
    for name, t in tensors.items():
        if t is None:
            continue
        at = t.get_device()
        if at < 0:
            raise ValueError(f"{fn}: {name} is not a GPU tensor")
        if dev < 0:
            dev = _current()
        if at != dev:
            raise ValueError(f"{fn}: {name} is on cuda:{at}, the current device is cuda:{dev}")


def _int32(fn: str, count: int | None = None, **tensors):
    """The named tensors are contiguous int32 tensors of `count` elements (any number: None)."""
    global _int32_type
    if _int32_type is None:
        import torch

        _int32_type = torch.int32
    for name, t in tensors.items():
        if t.dtype != _int32_type or not t.is_contiguous():
            raise ValueError(f"{fn}: {name} must be a contiguous int32 tensor")
        if count is not None and t.numel() != count:
            raise ValueError(f"{fn}: {name} needs {count} elements, not {t.numel()}")


class PagePool:
    """Free pages of a pool of n_pages pages as kv_page_map and kv_page_release keep them: a stack `free` and
    its height `count` (device int32).  A new pool is all free, page 0 on top."""

    def __init__(self, n_pages: int, device="cuda"):
        import torch

        self.n_pages = int(n_pages)
        self.free = torch.arange(self.n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        self.count = torch.full((1,), self.n_pages, dtype=torch.int32, device=device)

    def struct(self) -> PagePoolStruct:
        return PagePoolStruct(_ptr(self.free), _ptr(self.count), self.n_pages)


def kv_page_map(held, add, pool: PagePool, pages, page_size: int, cu, lens, pos, slots, err_flag=None, stream=None):
    """Tables and slots of one step: row b holds held[b] positions and adds add[b] tokens (int32 [B]).  Takes the
    new pages off `pool` into the table `pages` [B][max_pages] and writes lens [B] (may be held), cu [B + 1], and
    for the packed tokens pos [N] and slots [N] (-1 behind the last one).  A step that runs out of pages
    (CG_FLAG_POOL_EMPTY) is not repeated: the rows with a hole (-1) are released whole and begun again."""
    _on_device("kv_page_map", held=held, add=add, free=pool.free, count=pool.count, pages=pages, cu=cu, lens=lens,
               pos=pos, slots=slots, err_flag=err_flag)
    B, N = held.numel(), pos.numel()
    if pages.dim() != 2 or pages.shape[0] != B:
        raise ValueError("kv_page_map: pages must be [B][max_pages]")
    _int32("kv_page_map", B, held=held, add=add, lens=lens)
    _int32("kv_page_map", B + 1, cu=cu)
    _int32("kv_page_map", N, pos=pos, slots=slots)
    _int32("kv_page_map", None, pages=pages)
    ps = pool.struct()
    rc = lib().kv_page_map(_ptr(held), _ptr(add), B, C.byref(ps), _ptr(pages), pages.shape[1], page_size, N, _ptr(cu),
                           _ptr(lens), _ptr(pos), _ptr(slots), _ptr(err_flag), _stream(stream))
    _check("kv_page_map", rc)


def kv_page_release(lens, done, pool: PagePool, pages, page_size: int, err_flag=None, stream=None):
    """Rows with done[b] != 0 (int32 [B]) give their pages back to `pool`; their lens become 0."""
    _on_device("kv_page_release", lens=lens, done=done, free=pool.free, count=pool.count, pages=pages,
               err_flag=err_flag)
    B = lens.numel()
    if pages.dim() != 2 or pages.shape[0] != B:
        raise ValueError("kv_page_release: pages must be [B][max_pages]")
    _int32("kv_page_release", B, lens=lens, done=done)
    _int32("kv_page_release", None, pages=pages)
    ps = pool.struct()
    rc = lib().kv_page_release(_ptr(lens), _ptr(done), B, C.byref(ps), _ptr(pages), pages.shape[1], page_size,
                               _ptr(err_flag), _stream(stream))
    _check("kv_page_release", rc)


def rope_make(d_rot: int, layout: int = ROPE_HALF, base: float = 10000.0, scaling: int = ROPE_NONE, factor: float = 1.0,
              low: float = 1.0, high: float = 4.0, train_len: int = 0, amplitude: float = 1.0) -> RopePlan:
    """Plan of a rotation of the channels [0, d_rot): pairs (i, i + d_rot / 2) or neighbours, frequencies
    base^(-2 i / d_rot), for long contexts divided by `factor` (ROPE_LINEAR) or by the turns that a pair makes over
    train_len positions, from `low` turns (divided) to `high` (kept) (ROPE_RAMP)."""
    r = Rope(d_rot, layout, scaling, train_len, base, factor, low, high, amplitude)
    plan = RopePlan()
    _check("rope_make", lib().rope_make(C.byref(r), C.byref(plan)))
    return plan


def kv_rope(plan: RopePlan, x, y, pos, x2=None, y2=None, inverse: bool = False, stream=None):
    """y = x [L][B][H][T][d] turned by the tokens' positions pos (int32 [B][T]; negative: left as it was), x2 into
    y2 by the same launch; y may be x.  inverse: the transposed map (the gradient with respect to x)."""
    _on_device("kv_rope", x=x, y=y, x2=x2, y2=y2, pos=pos)
    _int32("kv_rope", x.shape[1] * x.shape[3], pos=pos)
    xv, yv = view(x), view(y)
    x2v = None if x2 is None else C.byref(view(x2))
    y2v = None if y2 is None else C.byref(view(y2))
    rc = lib().kv_rope(C.byref(plan), C.byref(xv), C.byref(yv), x2v, y2v, _ptr(pos), int(inverse), _stream(stream))
    _check("kv_rope", rc)


def kv_append_slots(l0: int, l1: int, k_new, v_new, slots, G_dev, shp: GaugeShape, codec: Codec, kc: Cache, vc: Cache,
                    err_flag=None, stream=None):
    """Encodes packed tokens k_new, v_new [l1-l0][1][H][N][d] into the page pools kc, vc at slots (int32 [N], as
    kv_page_map writes them; negative: skipped)."""
    _on_device("kv_append_slots", k_new=k_new, v_new=v_new, slots=slots, G_dev=G_dev, codes=kc.codes, v_codes=vc.codes,
               err_flag=err_flag)
    _int32("kv_append_slots", k_new.shape[3], slots=slots)
    kn, vn, cs, kcs, vcs = view(k_new), view(v_new), codec.struct(), kc.struct(), vc.struct()
    rc = lib().kv_append_slots(l0, l1, C.byref(kn), C.byref(vn), _ptr(slots), _ptr(G_dev), shp, C.byref(cs),
                               C.byref(kcs), C.byref(vcs), _ptr(err_flag), _stream(stream))
    _check("kv_append_slots", rc)


def attend_chunk_workspace_bytes(shp: GaugeShape, nl: int, N: int, B: int, max_q: int, Hq: int, max_pages: int,
                                 page_size: int, window: int = 0, sinks: int = 0) -> int:
    """Bytes of the kv_attend_chunk_paged call with exactly these arguments; fewer tokens or rows may need more."""
    return int(lib().attend_chunk_workspace_bytes(shp, nl, N, B, max_q, Hq, max_pages, page_size, window, sinks))


def attend_chunk_workspace_limit(shp: GaugeShape, nl: int, N: int, B: int, Hq: int, max_pages: int, page_size: int) -> int:
    """Bytes that every kv_attend_chunk_paged call of at most these sizes stays within: for a workspace kept across calls."""
    return int(lib().attend_chunk_workspace_limit(shp, nl, N, B, Hq, max_pages, page_size))


def kv_attend_chunk_paged(l0: int, l1: int, q, cu, max_q: int, kc: Cache, vc: Cache, pt: PageTable, G_dev,
                          shp: GaugeShape, codec: Codec, lens, scale: float, out, window: int = 0, sinks: int = 0,
                          workspace=None, err_flag=None, stream=None):
    """Attention of the packed new tokens q [l1-l0][1][Hq][N][d] (row b's: cu[b] .. cu[b+1], at most max_q) over
    page pools that hold them, causal or with a sliding window behind which the first `sinks` positions stay
    visible; lens: int32 [B] positions held with the new tokens.  Writes out (q's shape)."""
    _on_device("kv_attend_chunk_paged", q=q, cu=cu, codes=kc.codes, v_codes=vc.codes, G_dev=G_dev, lens=lens, out=out,
               workspace=workspace, err_flag=err_flag)
    B = lens.numel()
    _int32("kv_attend_chunk_paged", B, lens=lens)
    _int32("kv_attend_chunk_paged", B + 1, cu=cu)
    table = getattr(pt, "tensor", None)
    if table is not None:
        _on_device("kv_attend_chunk_paged", pages=table)
        if table.shape[0] != B:
            raise ValueError(f"kv_attend_chunk_paged: a page table of {table.shape[0]} rows, {B} lens")
    qv, ov, cs, kcs, vcs = view(q), view(out), codec.struct(), kc.struct(), vc.struct()
    if workspace is not None:
        need = attend_chunk_workspace_bytes(shp, l1 - l0, qv.T, B, max_q, qv.H, pt.max_pages, pt.page_size, window, sinks)
        if workspace.nbytes < need:
            raise ValueError(f"kv_attend_chunk_paged: workspace of {workspace.nbytes} bytes, {need} needed")
    rc = lib().kv_attend_chunk_paged(l0, l1, C.byref(qv), _ptr(cu), B, max_q, C.byref(kcs), C.byref(vcs), C.byref(pt),
                                     _ptr(G_dev), shp, C.byref(cs), _ptr(lens), float(scale), window, sinks,
                                     C.byref(ov), _ptr(workspace), _ptr(err_flag), _stream(stream))
    _check("kv_attend_chunk_paged", rc)


# ------------------------------------------------------------------------------------------
# a step that checks trees of drafted tokens
# ------------------------------------------------------------------------------------------

def kv_page_trim(lens, keep, pool: PagePool, pages, page_size: int, err_flag=None, stream=None):
    """Row b keeps its first keep[b] positions (int32 [B]): the pages past them go back to `pool`, lens[b] becomes keep[b]."""
    _on_device("kv_page_trim", lens=lens, keep=keep, free=pool.free, count=pool.count, pages=pages, err_flag=err_flag)
    B = lens.numel()
    if pages.dim() != 2 or pages.shape[0] != B:
        raise ValueError("kv_page_trim: pages must be [B][max_pages]")
    _int32("kv_page_trim", B, lens=lens, keep=keep)
    _int32("kv_page_trim", None, pages=pages)
    ps = pool.struct()
    rc = lib().kv_page_trim(_ptr(lens), _ptr(keep), B, C.byref(ps), _ptr(pages), pages.shape[1], page_size, _ptr(err_flag),
                            _stream(stream))
    _check("kv_page_trim", rc)


_int64_type = None


def _mask(fn: str, mask, N: int) -> int:
    """Words of a token's mask: a contiguous int64 tensor [N][words]."""
    global _int64_type
    if _int64_type is None:
        import torch

        _int64_type = torch.int64
    if mask.dtype != _int64_type or mask.dim() != 2 or mask.shape[0] != N or not mask.is_contiguous():
        raise ValueError(f"{fn}: mask must be a contiguous int64 tensor [{N}][words]")
    return mask.shape[1]


def kv_tree_map(parent, cu, lens, pos, mask, err_flag=None, stream=None, window: int = 0, sinks: int = 0):
    """Positions pos (int32 [N]) and masks (int64 [N][words]: bit j mod 64 of word j / 64 for the node itself and its
    ancestors) of the packed trees whose nodes' parents (int32 [N], indices within the row, -1: a root) are `parent`;
    row b's nodes are cu[b] .. cu[b + 1], the last of its lens[b] positions.  window, sinks: those of the attention that
    reads the masks; an ancestor `window` or more positions before its node is left out unless its position is below `sinks`."""
    _on_device("kv_tree_map", parent=parent, cu=cu, lens=lens, pos=pos, mask=mask, err_flag=err_flag)
    B, N = lens.numel(), parent.numel()
    _int32("kv_tree_map", N, parent=parent, pos=pos)
    _int32("kv_tree_map", B, lens=lens)
    _int32("kv_tree_map", B + 1, cu=cu)
    words = _mask("kv_tree_map", mask, N)
    rc = lib().kv_tree_map_window(_ptr(parent), _ptr(cu), _ptr(lens), B, N, words, window, sinks, _ptr(pos), _ptr(mask),
                                  _ptr(err_flag), _stream(stream))
    _check("kv_tree_map", rc)


def kv_append_rope(l0: int, l1: int, plan: RopePlan, k_new, v_new, pos, slots, G_dev, shp: GaugeShape, codec: Codec,
                   kc: Cache, vc: Cache, q=None, q_out=None, err_flag=None, stream=None):
    """Encodes packed tokens k_new, v_new [l1-l0][1][H][N][d] into the page pools kc, vc at slots (int32 [N]; negative:
    skipped), the keys turned by pos (int32 [N]; negative: the token is left out) before the gauge, and turns q
    [l1-l0][1][Hq][N][d] into q_out (may be q)."""
    _on_device("kv_append_rope", k_new=k_new, v_new=v_new, pos=pos, slots=slots, G_dev=G_dev, codes=kc.codes, v_codes=vc.codes,
               q=q, q_out=q_out, err_flag=err_flag)
    _int32("kv_append_rope", k_new.shape[3], pos=pos, slots=slots)
    kn, vn, cs, kcs, vcs = view(k_new), view(v_new), codec.struct(), kc.struct(), vc.struct()
    qv = None if q is None else C.byref(view(q))
    qo = None if q_out is None else C.byref(view(q_out))
    rc = lib().kv_append_rope(l0, l1, C.byref(plan), C.byref(kn), C.byref(vn), qv, qo, _ptr(pos), _ptr(slots), _ptr(G_dev),
                              shp, C.byref(cs), C.byref(kcs), C.byref(vcs), _ptr(err_flag), _stream(stream))
    _check("kv_append_rope", rc)


def attend_tree_workspace_bytes(shp: GaugeShape, nl: int, N: int, B: int, Hq: int, max_pages: int, page_size: int) -> int:
    """Bytes that every kv_attend_tree_paged call of at most these sizes stays within."""
    return int(lib().attend_tree_workspace_bytes(shp, nl, N, B, Hq, max_pages, page_size))


def kv_attend_tree_paged(l0: int, l1: int, q, cu, max_q: int, mask, kc: Cache, vc: Cache, pt: PageTable, G_dev,
                         shp: GaugeShape, codec: Codec, lens, scale: float, out, pos=None, window: int = 0, sinks: int = 0,
                         workspace=None, err_flag=None, stream=None):
    """Attention of the packed tokens q [l1-l0][1][Hq][N][d] (row b's: cu[b] .. cu[b+1], at most max_q) over page pools that
    hold them: all of what the row held before them (behind a window by the tokens' pos, int32 [N], the first `sinks` stay
    visible) and of its new tokens those whose bits are set in a token's mask (int64 [N][words]; with a window made by
    kv_tree_map with the same window and sinks); lens: int32 [B] positions held with the new tokens.  Writes out (q's shape)."""
    _on_device("kv_attend_tree_paged", q=q, cu=cu, mask=mask, pos=pos, codes=kc.codes, v_codes=vc.codes, G_dev=G_dev, lens=lens,
               out=out, workspace=workspace, err_flag=err_flag)
    B = lens.numel()
    _int32("kv_attend_tree_paged", B, lens=lens)
    _int32("kv_attend_tree_paged", B + 1, cu=cu)
    qv, ov, cs, kcs, vcs = view(q), view(out), codec.struct(), kc.struct(), vc.struct()
    words = _mask("kv_attend_tree_paged", mask, qv.T)
    if pos is not None:
        _int32("kv_attend_tree_paged", qv.T, pos=pos)
    table = getattr(pt, "tensor", None)
    if table is not None:
        _on_device("kv_attend_tree_paged", pages=table)
        if table.shape[0] != B:
            raise ValueError(f"kv_attend_tree_paged: a page table of {table.shape[0]} rows, {B} lens")
    if workspace is not None:
        need = attend_tree_workspace_bytes(shp, l1 - l0, qv.T, B, qv.H, pt.max_pages, pt.page_size)
        if workspace.nbytes < need:
            raise ValueError(f"kv_attend_tree_paged: workspace of {workspace.nbytes} bytes, {need} needed")
    rc = lib().kv_attend_tree_paged(l0, l1, C.byref(qv), _ptr(cu), B, max_q, _ptr(mask), words, _ptr(pos), C.byref(kcs),
                                    C.byref(vcs), C.byref(pt), _ptr(G_dev), shp, C.byref(cs), _ptr(lens), float(scale), window,
                                    sinks, C.byref(ov), _ptr(workspace), _ptr(err_flag), _stream(stream))
    _check("kv_attend_tree_paged", rc)


def kv_tree_accept(parent, cu, draft, target, path, kept, next, head=None, err_flag=None, stream=None):
    """Greedy check of packed trees: from each row's root on the lowest child whose draft (int32 [N]) is the model's choice
    (target, int32 [N]) after its parent; head: its choice before the roots (int32 [B]; None: the first root is kept).
    Writes the kept nodes to path (int32 [N], -1 behind them), their number to kept and the choice after them to next (int32 [B])."""
    _on_device("kv_tree_accept", parent=parent, cu=cu, draft=draft, target=target, path=path, kept=kept, next=next, head=head,
               err_flag=err_flag)
    B, N = kept.numel(), parent.numel()
    _int32("kv_tree_accept", N, parent=parent, draft=draft, target=target, path=path)
    _int32("kv_tree_accept", B, kept=kept, next=next)
    _int32("kv_tree_accept", B + 1, cu=cu)
    if head is not None:
        _int32("kv_tree_accept", B, head=head)
    rc = lib().kv_tree_accept(_ptr(parent), _ptr(cu), _ptr(draft), _ptr(target), _ptr(head), B, N, _ptr(path), _ptr(kept),
                              _ptr(next), _ptr(err_flag), _stream(stream))
    _check("kv_tree_accept", rc)


def kv_tree_keep(l0: int, l1: int, path, kept, cu, lens, pt: PageTable, codec: Codec, kc: Cache, vc: Cache, held,
                 err_flag=None, stream=None):
    """Moves the entries of each row's kept nodes (path, kept: as kv_tree_accept writes them) of both pools to the first places
    behind what the row held before its cu[b + 1] - cu[b] nodes; held (int32 [B], a buffer of its own) becomes the positions it
    then holds, for kv_page_trim (lens stay as they are)."""
    _on_device("kv_tree_keep", path=path, kept=kept, cu=cu, lens=lens, held=held, codes=kc.codes, v_codes=vc.codes,
               err_flag=err_flag)
    B, N = lens.numel(), path.numel()
    _int32("kv_tree_keep", N, path=path)
    _int32("kv_tree_keep", B, kept=kept, lens=lens, held=held)
    _int32("kv_tree_keep", B + 1, cu=cu)
    table = getattr(pt, "tensor", None)
    if table is not None:
        _on_device("kv_tree_keep", pages=table)
        if table.shape[0] != B:
            raise ValueError(f"kv_tree_keep: a page table of {table.shape[0]} rows, {B} lens")
    cs, kcs, vcs = codec.struct(), kc.struct(), vc.struct()
    # (no gauge is read: any group size says the pools' shape)
    shp = GaugeShape(kc.L, kc.H, kc.d, kc.d)
    rc = lib().kv_tree_keep(l0, l1, _ptr(path), _ptr(kept), _ptr(cu), _ptr(lens), B, N, C.byref(pt), shp, C.byref(cs),
                            C.byref(kcs), C.byref(vcs), _ptr(held), _ptr(err_flag), _stream(stream))
    _check("kv_tree_keep", rc)
