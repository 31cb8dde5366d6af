"""Python binding of liblamp.so (the C ABI declared in include/lamp.h).

Argument marshalling only: every step of the forward pass runs in the HIP
kernels of the library.  PyTorch provides device memory and the stream.  The
library must have been built (python -m paper_2609_39361_amd.build); there is
no fallback path.
"""
import collections
import ctypes
import functools
import math
import os
import struct

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# LAMP_LIBRARY may name the measurement build liblamp_phase.so (phase timer)
LIB_PATH = os.environ.get("LAMP_LIBRARY") or os.path.join(HERE, "liblamp.so")

LAMP_OK = 0
LAMP_ERR_NONFINITE_INPUT = 5
LAMP_ERR_WORKSPACE = 6
MASK_LOW, MASK_STAGE1, MASK_STAGE2, MASK_INACTIVE = 0, 1, 2, 3

# statistics words (include/lamp.h, LAMP_STAT_*)
STAT_NAMES = ("tiles", "stage1", "stage2", "inactive", "sat8", "sat16", "spec_unused", "late16")
STAT_HIST = len(STAT_NAMES)


def stats_words(nk):
    """Number of uint64 statistics words for nk sub-blocks per tile."""
    return STAT_HIST + nk + 1


class FwdExtra(ctypes.Structure):
    """struct lamp_fwd_extra (include/lamp.h)."""
    _fields_ = [("stats", ctypes.c_void_p), ("dbg_y8", ctypes.c_void_p), ("dbg_y16", ctypes.c_void_p),
                ("dbg_qb0", ctypes.c_int), ("dbg_nqb", ctypes.c_int), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class LampError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("lamp status %d: %s" % (status, msg))
        self.status = status


_lib = None


def lib():
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("liblamp.so is not built; run `python -m paper_2609_39361_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, f64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_size_t
        L.lamp_attn_fwd.argtypes = [P, P, P] + [i32] * 5 + [i32] * 5 + [f64, f64, ctypes.c_uint, P, P, P, P, P]
        L.lamp_attn_fwd.restype = i32
        L.lamp_attn_logits8.argtypes = [P, P] + [i32] * 9 + [P, P]
        L.lamp_attn_logits8.restype = i32
        L.lamp_attn_fwd_sr.argtypes = ([P, P, P] + [i32] * 5 + [i32] * 5 + [f64, f64, ctypes.c_uint, ctypes.c_uint64]
                                       + [P, P, P, P, P])
        L.lamp_attn_fwd_sr.restype = i32
        L.lamp_attn_fwd_noalloc.argtypes = [P, P, P] + [i32] * 5 + [i32] * 5 + [f64, f64, ctypes.c_uint, P, P, P, P, P]
        L.lamp_attn_fwd_noalloc.restype = i32
        L.lamp_attn_logits8_sr.argtypes = [P, P] + [i32] * 9 + [ctypes.c_uint64, P, P]
        L.lamp_attn_logits8_sr.restype = i32
        L.lamp_attn_logits16.argtypes = [P, P] + [i32] * 9 + [P, P]
        L.lamp_attn_logits16.restype = i32
        L.lamp_attn_decode.argtypes = [P, P, P] + [i32] * 9 + [f64, f64, ctypes.c_uint, P, P, P, P, P]
        L.lamp_attn_decode.restype = i32
        L.lamp_attn_logits_sim.argtypes = [P, P] + [i32] * 10 + [P, P]
        L.lamp_attn_logits_sim.restype = i32
        i64 = ctypes.c_int64
        L.lamp_qk_norm_rope.argtypes = [P, P, i32, i32, i32, i32, P, P, ctypes.c_uint, P, i32, i32, P, f64, P]
        L.lamp_qk_norm_rope.restype = i32
        L.lamp_kv_append.argtypes = [P, P, i32, i64, i64, i64, i64, P, P, P, i32, P, i32, i32, f64, P]
        L.lamp_kv_append.restype = i32
        L.lamp_attn_cache.argtypes = [P, i64, i64, i32, P, P, i32, i32, f64, P, P, P, sz, P]
        L.lamp_attn_cache.restype = i32
        L.lamp_attn_cache_workspace_size.argtypes = [i32] * 7
        L.lamp_attn_cache_workspace_size.restype = sz
        L.lamp_kv_advance.argtypes = [P, P, P, P, i64, i32, i32, i32, i32, P, i32, P, P, P, P, P, P]
        L.lamp_kv_advance.restype = i32
        L.lamp_kv_bounds.argtypes = [P, P, P, P]
        L.lamp_kv_bounds.restype = i32
        L.lamp_select_pages.argtypes = [P, i64, i64, i32, P, P, P, i32, i32, i32, P, P, sz, P]
        L.lamp_select_pages.restype = i32
        L.lamp_select_pages_workspace_size.argtypes = [i32] * 7
        L.lamp_select_pages_workspace_size.restype = sz
        L.lamp_attn_pages.argtypes = [P, i64, i64, i32, P, P, P, i32, f64, P, P, P, sz, P]
        L.lamp_attn_pages.restype = i32
        L.lamp_attn_pages_workspace_size.argtypes = [i32] * 6
        L.lamp_attn_pages_workspace_size.restype = sz
        L.lamp_attn_shared.argtypes = [P, i64, i64, i32, P, P, P, P, i32, f64, P, P, P, sz, P]
        L.lamp_attn_shared.restype = i32
        L.lamp_attn_shared_workspace_size.argtypes = [i32] * 8
        L.lamp_attn_shared_workspace_size.restype = sz
        L.lamp_get_sim_tables.argtypes = [i32, P, P]
        L.lamp_get_sim_tables.restype = i32
        L.lamp_attn_fwd_workspace_size.argtypes = [i32] * 8
        L.lamp_attn_fwd_workspace_size.restype = sz
        L.lamp_attn_decode_workspace_size.argtypes = [i32] * 6
        L.lamp_attn_decode_workspace_size.restype = sz
        L.lamp_reserve.argtypes = [i32, sz]
        L.lamp_reserve.restype = i32
        L.lamp_init.argtypes = [i32]
        L.lamp_init.restype = i32
        L.lamp_shutdown.argtypes = []
        L.lamp_shutdown.restype = None
        L.lamp_selftest_e4m3.argtypes = [P, P, P, sz, P]
        L.lamp_selftest_e4m3.restype = i32
        L.lamp_selftest_exp_doc.argtypes = [P, P, sz, P]
        L.lamp_selftest_exp_doc.restype = i32
        L.lamp_get_tables.argtypes = [i32, P, P]
        L.lamp_get_tables.restype = i32
        L.lamp_get_exp16_parts.argtypes = [i32, P]
        L.lamp_get_exp16_parts.restype = i32
        L.lamp_issue_rates.argtypes = [P, P]
        L.lamp_issue_rates.restype = i32
        L.lamp_phase_read.argtypes = [P, i32]
        L.lamp_phase_read.restype = i32
        L.lamp_timing_enable.argtypes = [i32]
        L.lamp_timing_enable.restype = i32
        L.lamp_timing_read.argtypes = [P, P, P]
        L.lamp_timing_read.restype = i32
        L.lamp_status_str.argtypes = [i32]
        L.lamp_status_str.restype = ctypes.c_char_p
        L.lamp_last_error.argtypes = []
        L.lamp_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(rc):
    if rc != LAMP_OK:
        L = lib()
        raise LampError(rc, "%s: %s" % (L.lamp_status_str(rc).decode(), L.lamp_last_error().decode()))


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _stream(device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _check_inputs(q, k, v=None):
    for t in (q, k) + ((v,) if v is not None else ()):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError("q, k, v must be contiguous 4-d bf16 CUDA tensors [B,H,N,d]")
    B, Hq, N, d = q.shape
    if k.shape[0] != B or k.shape[2] != N or k.shape[3] != d:
        raise ValueError("k shape %s does not match q %s" % (tuple(k.shape), tuple(q.shape)))
    if v is not None and v.shape != k.shape:
        raise ValueError("v shape %s differs from k %s" % (tuple(v.shape), tuple(k.shape)))
    if q.device != k.device or (v is not None and v.device != q.device):
        raise ValueError("q, k, v must be on one device")
    return B, Hq, k.shape[1], N, d


STAGE1_OFF = 1   # the first stage disabled: mu_hat from the 8-bit maxima, stage 2 alone recomputes
MU_TRUNC = 2     # 8-bit shifts against mu_hat truncated to e4m3 (SIM profile: to 3 mantissa bits)
SIM_PROFILE = 4  # the SIM precision profile (FP32 range, 3 / 11 mantissa bits, no saturation)
CHECK_FINITE = 8  # check q, k, v for NaN / infinity first (synchronous; LAMP_ERR_NONFINITE_INPUT)
COMPACT = 16     # the compact register layout of Sec. 3.3 as the kernel's schedule (same results)
# attn_decode flag: one key chunk and the passes one after another instead of the key-chunk
# pipeline (same masks and lse; O equal up to the order of its final sums)
DECODE_SERIAL = 256


def _check_out(t, name, shape, dtype, device):
    if (not isinstance(t, torch.Tensor) or tuple(t.shape) != tuple(shape) or t.dtype != dtype
            or t.device != device or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s" % (name, dtype, tuple(shape), device))


def _extra(stats=None, observe=None, workspace=None, device=None, nk=4):
    """(FwdExtra or None, tensors kept alive) from the optional arguments."""
    if stats is None and observe is None and workspace is None:
        return None, ()
    e = FwdExtra()
    keep = []
    if stats is not None:
        _check_out(stats, "stats", (stats_words(nk),), torch.int64, device)
        e.stats = stats.data_ptr()
        keep.append(stats)
    if observe is not None:
        qb0, nqb, y8, y16 = observe
        e.dbg_qb0, e.dbg_nqb = int(qb0), int(nqb)
        for t in (y8, y16):
            if t is not None:
                if not t.is_contiguous() or t.device != device:
                    raise ValueError("observable arrays must be contiguous tensors on the inputs' device")
                keep.append(t)
        e.dbg_y8 = y8.data_ptr() if y8 is not None else None
        e.dbg_y16 = y16.data_ptr() if y16 is not None else None
    if workspace is not None:
        if workspace.device != device or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the inputs' device")
        e.workspace = workspace.data_ptr()
        e.workspace_bytes = workspace.numel() * workspace.element_size()
        keep.append(workspace)
    return e, tuple(keep)


def attn_fwd(q, k, v, causal=True, window=0, bq=128, bk=16, nk=4, delta=2.0 ** -8, tau=0.5, out=None, flags=0,
             sr_seed=None, stats=None, observe=None, workspace=None):
    """LampAttention forward pass.  Returns (o fp32 [B,Hq,N,d], lse fp32
    [B,Hq,N], mask uint8 [B,Hq,ceil(N/bq),ceil(N/(bk*nk))*nk]); N need not be
    a multiple of the block sizes.  `out` may supply those three tensors to
    write into; `flags` selects the variants STAGE1_OFF, MU_TRUNC, the
    SIM_PROFILE numerics and the CHECK_FINITE input check.  With `sr_seed` (an
    int below 2^64) the 8-bit accumulation is rounded stochastically with that
    seed (lamp_attn_fwd_sr).

    Optional (struct lamp_fwd_extra): `stats`, an int64 tensor of
    stats_words(nk) elements on the device that the call adds the statistics
    words to; `observe` = (qb0, nqb, y8, y16), the forward kernel's 8-bit and
    16-bit logit codes of query blocks [qb0, qb0+nqb) (see observe_logits);
    `workspace`, a device tensor of at least fwd_workspace_size(...) bytes."""
    B, Hq, Hkv, N, d = _check_inputs(q, k, v)
    dev = q.device
    mshape = (B, Hq, -(-N // bq), -(-N // (bk * nk)) * nk)
    if out is None:
        o = torch.empty((B, Hq, N, d), dtype=torch.float32, device=dev)
        lse = torch.empty((B, Hq, N), dtype=torch.float32, device=dev)
        mask = torch.empty(mshape, dtype=torch.uint8, device=dev)
    else:
        o, lse, mask = out
        _check_out(o, "o", (B, Hq, N, d), torch.float32, dev)
        _check_out(lse, "lse", (B, Hq, N), torch.float32, dev)
        _check_out(mask, "mask", mshape, torch.uint8, dev)
    extra, keep = _extra(stats, observe, workspace, dev, nk)
    ep = ctypes.byref(extra) if extra is not None else None
    with torch.cuda.device(dev):
        if sr_seed is None:
            rc = lib().lamp_attn_fwd(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, N, d, int(causal), int(window),
                                     bq, bk, nk, float(delta), float(tau), int(flags), _ptr(o), _ptr(lse), _ptr(mask),
                                     ep, _stream(dev))
        else:
            rc = lib().lamp_attn_fwd_sr(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, N, d, int(causal), int(window),
                                        bq, bk, nk, float(delta), float(tau), int(flags), int(sr_seed),
                                        _ptr(o), _ptr(lse), _ptr(mask), ep, _stream(dev))
    del keep
    _check(rc)
    return o, lse, mask


NOALLOC_SCRATCH_BYTES = 256 << 20


def attn_fwd_noalloc(q, k, v, out, causal=True, window=0, bq=128, bk=16, nk=4, delta=2.0 ** -8, tau=0.5, flags=0,
                     stats=None):
    """attn_fwd through lamp_attn_fwd_noalloc: the library allocates nothing
    (its workspace is the device's fixed scratch of NOALLOC_SCRATCH_BYTES;
    init(device) must have been called).  `out` = (o, lse, mask) as for
    attn_fwd is required, so that nothing is allocated here either."""
    B, Hq, Hkv, N, d = _check_inputs(q, k, v)
    dev = q.device
    o, lse, mask = out
    _check_out(o, "o", (B, Hq, N, d), torch.float32, dev)
    _check_out(lse, "lse", (B, Hq, N), torch.float32, dev)
    _check_out(mask, "mask", (B, Hq, -(-N // bq), -(-N // (bk * nk)) * nk), torch.uint8, dev)
    extra, keep = _extra(stats=stats, device=dev, nk=nk)
    ep = ctypes.byref(extra) if extra is not None else None
    with torch.cuda.device(dev):
        rc = lib().lamp_attn_fwd_noalloc(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, N, d, int(causal), int(window),
                                         bq, bk, nk, float(delta), float(tau), int(flags), _ptr(o), _ptr(lse),
                                         _ptr(mask), ep, _stream(dev))
    del keep
    _check(rc)
    return o, lse, mask


def observe_logits(q, k, v, qb0, nqb, causal=True, window=0, bq=128, bk=16, nk=4, delta=2.0 ** -8, tau=0.5,
                   flags=0, sr_seed=None, stats=None):
    """attn_fwd that also returns the forward kernel's own logit codes of the
    query blocks [qb0, qb0+nqb) of every (b, h): (o, lse, mask, y8, y16),
    y8 uint8 [B,Hq,nqb*bq,Nt] (e4m3 codes of visible pairs, 0xFF elsewhere)
    and y16 int16 bit patterns [B,Hq,nqb*bq,Nt] (e4m11 codes of visible pairs
    in 16-bit sub-blocks, 0xFFFF elsewhere), Nt = ceil(N/(bk*nk))*bk*nk."""
    B, Hq, Hkv, N, d = _check_inputs(q, k, v)
    Nt = -(-N // (bk * nk)) * bk * nk
    y8 = torch.empty((B, Hq, nqb * bq, Nt), dtype=torch.uint8, device=q.device)
    y16 = torch.empty((B, Hq, nqb * bq, Nt), dtype=torch.int16, device=q.device)
    o, lse, mask = attn_fwd(q, k, v, causal, window, bq, bk, nk, delta, tau, flags=flags, sr_seed=sr_seed,
                            stats=stats, observe=(qb0, nqb, y8, y16))
    return o, lse, mask, y8, y16


def fwd_workspace_size(B, Hq, Hkv, N, d, bq=128, bk=16, nk=4):
    """Bytes of workspace one attn_fwd call needs."""
    return int(lib().lamp_attn_fwd_workspace_size(B, Hq, Hkv, N, d, bq, bk, nk))


def decode_workspace_size(B, Hq, Hkv, M, N, d):
    return int(lib().lamp_attn_decode_workspace_size(B, Hq, Hkv, M, N, d))


def reserve(device, nbytes):
    """Grow the library's workspace of `device` to nbytes now (synchronous)."""
    _check(lib().lamp_reserve(int(device), int(nbytes)))


def stats_dict(stats, nk=4):
    """The statistics words as a dict (names of STAT_NAMES, 'hist' a list)."""
    w = [int(x) for x in stats.cpu().tolist()]
    r = dict(zip(STAT_NAMES, w[:STAT_HIST]))
    r["hist"] = w[STAT_HIST:STAT_HIST + nk + 1]
    return r


def attn_decode(q, k, v, causal=True, window=0, tk=64, delta=2.0 ** -8, tau=0.5, out=None, flags=0,
                workspace=None):
    """LampAttention in the vector form (Sec. 2, Eq. (6)) for M query rows per
    (b, h) at positions N-M .. N-1: q [B,Hq,M,d], k / v [B,Hkv,N,d] bf16.
    Returns (o fp32 [B,Hq,M,d], lse fp32 [B,Hq,M], mask uint8
    [B,Hq,M,ceil(N/tk)*tk] one code per key)."""
    if q.dim() != 4 or k.dim() != 4 or v.shape != k.shape:
        raise ValueError("q [B,Hq,M,d], k and v [B,Hkv,N,d] expected")
    B, Hq, M, d = q.shape
    Hkv, N = k.shape[1], k.shape[2]
    for t in (q, k, v):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("q, k, v must be contiguous bf16 CUDA tensors")
    dev = q.device
    if q.device != k.device or v.device != k.device:
        raise ValueError("q, k, v must be on one device")
    mshape = (B, Hq, M, -(-N // tk) * tk)
    if out is None:
        o = torch.empty((B, Hq, M, d), dtype=torch.float32, device=dev)
        lse = torch.empty((B, Hq, M), dtype=torch.float32, device=dev)
        mask = torch.empty(mshape, dtype=torch.uint8, device=dev)
    else:
        o, lse, mask = out
        _check_out(o, "o", (B, Hq, M, d), torch.float32, dev)
        _check_out(lse, "lse", (B, Hq, M), torch.float32, dev)
        _check_out(mask, "mask", mshape, torch.uint8, dev)
    extra, keep = _extra(workspace=workspace, device=dev)
    ep = ctypes.byref(extra) if extra is not None else None
    with torch.cuda.device(dev):
        rc = lib().lamp_attn_decode(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, M, N, d, int(causal), int(window), tk,
                                    float(delta), float(tau), int(flags), _ptr(o), _ptr(lse), _ptr(mask),
                                    ep, _stream(dev))
    del keep
    _check(rc)
    return o, lse, mask


# --- serving: norms with rotation, the 8-bit paged cache, attention over it ----
# A serving step makes these calls once a layer, so that the host's time counts:
# each has one test of everything a call must be, and names what is wrong only
# where that fails; the C structs are packed bytes.

_ROWS3 = struct.Struct("@" + "Pqqqi0P" * 3)   # struct lamp_rows [3] (include/lamp.h)
_CACHE = struct.Struct("@PPPPiiii")            # struct lamp_cache
_BATCH = struct.Struct("@PqPPiii0P")           # struct lamp_batch

# An 8-bit paged cache: codes k [pages,Hkv,page,d] and v [pages,Hkv,d,page] (float8_e4m3fn, V
# transposed within its page), scales k_scale and v_scale [pages,Hkv] (fp32 powers of two)
KVCache = collections.namedtuple("KVCache", "k v k_scale v_scale")

_BF16, _F32, _I32, _E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn
_FLOATS = (_BF16, _F32)


def kv_cache(pages, Hkv, d, page=64, device="cuda"):
    """An empty KVCache of `pages` pages of `page` tokens (zero codes and scales)."""
    z = dict(device=device)
    return KVCache(torch.zeros((pages, Hkv, page, d), dtype=torch.uint8, **z).view(_E4M3),
                   torch.zeros((pages, Hkv, d, page), dtype=torch.uint8, **z).view(_E4M3),
                   torch.zeros((pages, Hkv), dtype=_F32, **z), torch.zeros((pages, Hkv), dtype=_F32, **z))


def rope_table(n, rot, base=1e6, device="cuda"):
    """The rotation's table of positions 0 .. n-1: fp32 [n, rot], rot/2 cosines then rot/2 sines of
    position * base^(-2i/rot) (angles in fp64)."""
    inv = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    ang = torch.arange(n, dtype=torch.float64, device=device)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], dim=-1).float()


# (the calls behind torch's public ones, without the objects those make; a torch built without a GPU has none)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(dev, fn, *args):
    """One library call on the current stream of CUDA device `dev` (an index)."""
    if _current_device() == dev:
        rc = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc:
        _check(rc)


def _must(t, name, dtypes, dev, shape=None):
    """Refuses what is not a tensor of `dtypes` on CUDA device `dev`, contiguous in its last dimension (`shape`: of that
    shape, dense)."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.get_device() != dev or dev < 0:
        raise ValueError("%s must be a %s tensor on CUDA device %d" % (name, " or ".join(str(x) for x in dtypes), max(dev, 0)))
    if shape is not None and (tuple(t.shape) != tuple(shape) or not t.is_contiguous()):
        raise ValueError("%s must be contiguous, of shape %s" % (name, tuple(shape)))
    if t.dim() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)


def _gain(w, name, dev, d):
    """(pointer, whether fp32) of a gain."""
    if w is None:
        return None, 0
    if w.get_device() != dev or w.shape != (d,) or not w.is_contiguous() or w.dtype not in _FLOATS:
        _must(w, name, _FLOATS, dev, (d,))
    return w.data_ptr(), 1 if w.dtype is _F32 else 0


def _rope(rope, dev):
    """(pointer, positions, rotated channels) of a table."""
    if rope is None:
        return None, 0, 0
    if rope.dtype is not _F32 or rope.get_device() != dev or rope.dim() != 2 or not rope.is_contiguous():
        _must(rope, "rope", (_F32,), dev)
        raise ValueError("rope must be a contiguous [positions, rot] table")
    n, rot = rope.shape
    if n == 0 or rot == 0:   # (its address is null: "not rotated")
        raise ValueError("rope must have rows and channels, not shape %s" % ((n, rot),))
    return rope.data_ptr(), n, rot


def qk_norm_rope(q, k=None, v=None, q_weight=None, k_weight=None, rope=None, positions=None, eps=1e-6, out=None):
    """RMS norm of every query and key head by the gains q_weight / k_weight [d] (None: not normed), then
    the rotation by `rope` (a table as of rope_table, None: not rotated), in one pass.

    Inputs bf16 or fp32 (all the same), outputs bf16; the last dimension contiguous, rows of 16-byte
    alignment (slices of a fused projection are fine).  Prompts: q [B,N,Hq,d], k and v [B,N,Hkv,d] give
    [B,H,N,d], what attn_fwd reads.  Tokens of a serving step: q [T,Hq,d], k and v [T,Hkv,d] give [T,H,d].
    `positions`: int32 [B,N] or [T]; default 0 .. N-1.  v is laid out (and rounded) with them.  `out`: the
    tensors to write into (None where the input is None), of the outputs' shapes with any strides; tokens
    may be written in place.  Returns (q, k, v), None for what was not given."""
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() not in (3, 4) or q.dtype not in _FLOATS:
        raise ValueError("q must be a bf16 or fp32 CUDA tensor [B,N,Hq,d] or [T,Hq,d]")
    dev, shape, dtype = q.get_device(), q.shape, q.dtype
    if len(shape) == 4:
        B, N, Hq, d = shape
        prompt = True
    else:
        N, Hq, d = shape
        B, prompt = 1, False
    qw, q32 = _gain(q_weight, "q_weight", dev, d)
    kw, k32 = _gain(k_weight, "k_weight", dev, d)
    table, npos, rot = _rope(rope, dev)
    if positions is not None:
        if positions.dtype is not _I32 or positions.get_device() != dev or positions.shape != shape[:-2] \
                or not positions.is_contiguous():
            _must(positions, "positions", (_I32,), dev, shape[:-2])
    rows_in, rows_out, outs = [], [], []
    for i, t in enumerate((q, k, v)):
        o = None if out is None else out[i]
        if t is None:
            if o is not None:
                raise ValueError("out must hold one tensor for each input")
            rows_in += (0, 0, 0, 0, 0)
            rows_out += (0, 0, 0, 0, 0)
            outs.append(None)
            continue
        if i:
            if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != dev:
                _must(t, "qkv"[i], (dtype,), dev)
            if t.dim() != len(shape) or t.shape[:-2] != shape[:-2] or t.shape[-1] != d:
                raise ValueError("%s shape %s does not match q %s" % ("qkv"[i], tuple(t.shape), tuple(shape)))
        if t.stride(-1) != 1:
            _must(t, "qkv"[i], (dtype,), dev)
        H = t.shape[-2]
        want = (B, H, N, d) if prompt else (N, H, d)
        if o is None:
            if out is not None:
                raise ValueError("out must hold one tensor for each input")
            o = q.new_empty(want, dtype=_BF16)
        else:
            _must(o, "out[%d]" % i, (_BF16,), dev)
            if o.shape != want:
                raise ValueError("out[%d] must be of shape %s" % (i, want))
        outs.append(o)
        if prompt:
            b, n, h, _ = t.stride()
            rows_in += (t.data_ptr(), b, n, h, H)
            b, h, n, _ = o.stride()
        else:
            n, h, _ = t.stride()
            rows_in += (t.data_ptr(), 0, n, h, H)
            b, (n, h, _) = 0, o.stride()
        rows_out += (o.data_ptr(), b, n, h, H)
    if k is not None and v is not None and k.shape != v.shape:
        raise ValueError("v shape %s differs from k %s" % (tuple(v.shape), tuple(k.shape)))
    if B * N and d:
        _call(dev, lib().lamp_qk_norm_rope, _ROWS3.pack(*rows_in), _ROWS3.pack(*rows_out), B, N, d,
              1 if dtype is _F32 else 0, qw, kw, q32 + 2 * k32, table, npos, rot,
              None if positions is None else positions.data_ptr(), float(eps))
    return tuple(outs)


def _paged(cache, block_table, kv_lens, q_start, T):
    """(lamp_cache, lamp_batch, device, Hkv, page, d, S, width) of a call, checked."""
    kc, vc, ks, vs = cache
    if not isinstance(kc, torch.Tensor) or kc.dim() != 4 or not kc.is_cuda:
        raise ValueError("cache.k must be a float8_e4m3fn CUDA tensor [pages,Hkv,page,d]")
    dev = kc.get_device()
    pages, Hkv, page, d = kc.shape
    if not (kc.dtype is _E4M3 and vc.dtype is _E4M3 and ks.dtype is _F32 and vs.dtype is _F32
            and vc.get_device() == dev and ks.get_device() == dev and vs.get_device() == dev
            and vc.shape == (pages, Hkv, d, page) and ks.shape == (pages, Hkv) and vs.shape == (pages, Hkv)
            and kc.is_contiguous() and vc.is_contiguous() and ks.is_contiguous() and vs.is_contiguous()):
        _must(kc, "cache.k", (_E4M3,), dev, kc.shape)
        _must(vc, "cache.v", (_E4M3,), dev, (pages, Hkv, d, page))
        _must(ks, "cache.k_scale", (_F32,), dev, (pages, Hkv))
        _must(vs, "cache.v_scale", (_F32,), dev, (pages, Hkv))
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
        raise ValueError("block_table must be an int32 tensor [S, pages of a sequence]")
    S, width = block_table.shape
    if not (block_table.dtype is _I32 and kv_lens.dtype is _I32 and block_table.get_device() == dev
            and kv_lens.get_device() == dev and kv_lens.shape == (S,) and kv_lens.is_contiguous()
            and (width < 2 or block_table.stride(1) == 1)):
        _must(block_table, "block_table", (_I32,), dev)
        _must(kv_lens, "kv_lens", (_I32,), dev, (S,))
    if q_start is not None:
        if not (q_start.dtype is _I32 and q_start.get_device() == dev and q_start.shape == (S + 1,)
                and q_start.is_contiguous()):
            _must(q_start, "q_start", (_I32,), dev, (S + 1,))
    elif T != S:
        raise ValueError("without q_start there is one token for each of the %d sequences, not %d" % (S, T))
    return (_CACHE.pack(kc.data_ptr(), vc.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, Hkv, page, d),
            _BATCH.pack(block_table.data_ptr(), block_table.stride(0), kv_lens.data_ptr(),
                        0 if q_start is None else q_start.data_ptr(), S, T, width), dev, Hkv, page, d, S, width)


def kv_append(k, v, cache, block_table, kv_lens, q_start=None, k_weight=None, rope=None, eps=1e-6):
    """Append new keys and values [T,Hkv,d] (bf16 or fp32, token and head strides free) to a KVCache; the
    keys normed by k_weight and rotated by `rope` on the way (None: not), in fp32 with one rounding to e4m3.

    Sequence s has the tokens q_start[s] .. q_start[s+1]-1 (int32 [S+1]; None: token s alone), its length
    with them is kv_lens[s] (int32 [S]) and its pages are block_table[s] (int32 [S,width]).  A page's scale
    is the smallest power of two under which its largest element fits e4m3; when later tokens need a
    larger one, the codes there are rescaled.  Tokens without a page in the table are dropped.  All of it
    is read on the device, so that a captured call follows lengths that change.  Returns the cache."""
    if not isinstance(k, torch.Tensor) or not isinstance(v, torch.Tensor) or k.dim() != 3 or k.shape != v.shape:
        raise ValueError("k and v [T,Hkv,d] expected")
    T, H, dk = k.shape
    c, b, dev, Hkv, _, d, _, _ = _paged(cache, block_table, kv_lens, q_start, T)
    dtype = k.dtype
    if not (dtype in _FLOATS and v.dtype is dtype and k.get_device() == dev and v.get_device() == dev
            and k.stride(2) == 1 and v.stride(2) == 1):
        _must(k, "k", _FLOATS, dev)
        _must(v, "v", (dtype,), dev)
    if H != Hkv or dk != d:
        raise ValueError("k of %d heads and d = %d, a cache of %d and %d" % (H, dk, Hkv, d))
    w, w32 = _gain(k_weight, "k_weight", dev, d)
    _call(dev, lib().lamp_kv_append, k.data_ptr(), v.data_ptr(), 1 if dtype is _F32 else 0, *k.stride()[:2], *v.stride()[:2], c, b,
          w, w32, *_rope(rope, dev), float(eps))
    return cache


def attn_cache_workspace_size(T, S, Hq, Hkv, d, page, width):
    """Bytes of workspace one attn_cache call needs (0: none)."""
    return int(lib().lamp_attn_cache_workspace_size(T, S, Hq, Hkv, d, page, width))


def attn_cache(q, cache, block_table, kv_lens, q_start=None, causal=True, window=0, scale=None, out=None,
               workspace=None):
    """Softmax attention of new tokens q [T,Hq,d] (bf16, token and head strides free) over a KVCache that
    holds their own keys already: (o bf16 [T,Hq,d], lse fp32 [T,Hq]).

    block_table, kv_lens and q_start as for kv_append: prompts, chunks and single tokens of any lengths in
    one call.  The token at position p sees the sequence's keys j <= p (causal) with j > p - window
    (window > 0).  `scale` of the logits: default 1/sqrt(d).  A row that sees no key has o = 0 and
    lse = -inf (one whose logits are all -inf: o = NaN); tokens behind q_start[S] are left as they are in
    `out` = (o, lse).  `workspace`: a device
    tensor of attn_cache_workspace_size(...) bytes; by default one of torch's, on the current stream."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q [T,Hq,d] expected")
    T, Hq, dq = q.shape
    c, b, dev, Hkv, page, d, S, width = _paged(cache, block_table, kv_lens, q_start, T)
    if q.dtype is not _BF16 or q.get_device() != dev or q.stride(2) != 1:
        _must(q, "q", (_BF16,), dev)
    if dq != d:
        raise ValueError("q of d = %d, a cache of %d" % (dq, d))
    if out is None:
        o, lse = q.new_empty((T, Hq, d)), q.new_empty((T, Hq), dtype=_F32)
    else:
        o, lse = out
        _must(o, "o", (_BF16,), dev, (T, Hq, d))
        _must(lse, "lse", (_F32,), dev, (T, Hq))
    L = lib()
    if workspace is None:
        need = L.lamp_attn_cache_workspace_size(T, S, Hq, Hkv, d, page, width)
        if need:
            workspace = q.new_empty(need, dtype=torch.uint8)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the inputs' device")
    else:
        need = workspace.numel() * workspace.element_size()
        if not need and L.lamp_attn_cache_workspace_size(T, S, Hq, Hkv, d, page, width):   # (its address is null)
            raise ValueError("workspace is empty")
    window = max(-1, min(int(window), 0x7FFFFFFF))   # (no key lies farther back; ctypes would take the low 32 bits)
    _call(dev, L.lamp_attn_cache, q.data_ptr(), *q.stride()[:2], Hq, c, b, 1 if causal else 0, window,
          d ** -0.5 if scale is None else float(scale), o.data_ptr(), lse.data_ptr(),
          None if workspace is None else workspace.data_ptr(), need)
    return o, lse


# --- serving long contexts and changing batches ---------------------------------

# Free pages of a cache: ring int32 [pages]; state int32 [4]: the ring's first free entry, how many there are,
# the pages that the last step needed, and why it was not admitted (0: it was; include/lamp.h)
KVPool = collections.namedtuple("KVPool", "ring state")


def _c_int(x, name):
    """A size as the library takes it (ctypes would take the low 32 bits of others)."""
    x = int(x)
    if not -0x80000000 <= x <= 0x7FFFFFFF:
        raise ValueError("%s=%d is beyond a C int" % (name, x))
    return x


def kv_pool(pages, device="cuda"):
    """A KVPool in which the pages 0 .. pages-1 are free."""
    return KVPool(torch.arange(pages, dtype=_I32, device=device), torch.tensor([0, pages, 0, 0], dtype=_I32, device=device))


def kv_advance(pool, block_table, kv_lens, add, page, tokens, prefix_lens=None, out=None):
    """The next step of a batch, planned on the device: sequence s, of kv_lens[s] keys, adds add[s] tokens (int32 [S];
    negative: it leaves, and its pages go back to the pool).  Pages of `page` tokens for the new ones are taken from the
    pool and entered in block_table (int32 [S,width], in place).  Returns (kv_lens [S], q_start [S+1], positions [tokens],
    pool) as kv_append, qk_norm_rope and the attentions take them: the lengths with the new tokens, and 0 as the position
    of tokens behind the last.

    prefix_lens (int32 [S]): the first prefix_lens[s] // page places hold pages that the sequence shares; they do not go
    back.  A step with too few free pages, a sequence longer than the table or more than `tokens` new tokens adds no
    token; pool.state[3] says why.  `out` = (kv_lens, q_start, positions, state): tensors to write into, of which kv_lens
    and state may be the inputs, so that a captured call goes on from step to step."""
    ring, state = pool
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2 or not block_table.is_cuda:
        raise ValueError("block_table must be an int32 CUDA tensor [S, pages of a sequence]")
    dev = block_table.get_device()
    S, width = block_table.shape
    if not (block_table.dtype is _I32 and ring.dtype is _I32 and state.dtype is _I32 and kv_lens.dtype is _I32 and add.dtype is _I32
            and ring.get_device() == dev and state.get_device() == dev and kv_lens.get_device() == dev and add.get_device() == dev
            and state.shape == (4,) and kv_lens.shape == (S,) and add.shape == (S,) and ring.dim() == 1 and ring.is_contiguous()
            and state.is_contiguous() and kv_lens.is_contiguous() and add.is_contiguous() and (width < 2 or block_table.stride(1) == 1)):
        _must(block_table, "block_table", (_I32,), dev)
        _must(ring, "pool.ring", (_I32,), dev, (ring.numel(),))
        _must(state, "pool.state", (_I32,), dev, (4,))
        _must(kv_lens, "kv_lens", (_I32,), dev, (S,))
        _must(add, "add", (_I32,), dev, (S,))
    if S > 1 and block_table.stride(0) < width:   # (written to)
        raise ValueError("rows of block_table share memory")
    if prefix_lens is not None and (prefix_lens.dtype is not _I32 or prefix_lens.get_device() != dev or prefix_lens.shape != (S,)
                                    or not prefix_lens.is_contiguous()):
        _must(prefix_lens, "prefix_lens", (_I32,), dev, (S,))
    page, tokens = _c_int(page, "page"), _c_int(tokens, "tokens")
    if tokens < 0:
        raise ValueError("tokens must not be negative")
    if out is None:
        lens, q_start, positions, new_state = kv_lens.new_empty(2 * S + tokens + 5).split((S, S + 1, tokens, 4))
    else:
        lens, q_start, positions, new_state = out
        for t, name, n in ((lens, "kv_lens", S), (q_start, "q_start", S + 1), (positions, "positions", tokens),
                           (new_state, "state", 4)):
            _must(t, "out: " + name, (_I32,), dev, (n,))
    _call(dev, lib().lamp_kv_advance, kv_lens.data_ptr(), add.data_ptr(),
          None if prefix_lens is None else prefix_lens.data_ptr(), block_table.data_ptr(), block_table.stride(0), S, width,
          page, tokens, ring.data_ptr(), ring.numel(), state.data_ptr(), lens.data_ptr(), q_start.data_ptr(),
          positions.data_ptr(), new_state.data_ptr())
    return lens, q_start, positions, KVPool(ring, new_state)


def kv_page_bounds(cache):
    """Bounds of an empty KVCache's pages, for kv_bounds: int8 [pages,Hkv,2,d]."""
    pages, Hkv, _, d = cache.k.shape
    return torch.zeros((pages, Hkv, 2, d), dtype=torch.int8, device=cache.k.device)


def _bounds(bounds, dev, shape):
    if not isinstance(bounds, torch.Tensor) or bounds.dtype is not torch.int8 or bounds.get_device() != dev \
            or bounds.shape != shape or not bounds.is_contiguous():
        _must(bounds, "bounds", (torch.int8,), dev, shape)
    return bounds.data_ptr()


def kv_bounds(cache, bounds, block_table, kv_lens, tokens, q_start=None):
    """Bring `bounds` (of kv_page_bounds) up to date for the pages that a batch of `tokens` new tokens went to, after
    kv_append with the same block_table, kv_lens and q_start: the range of each channel over a page's keys in units of 4
    code values, bounds[:,:,0] the largest (rounded up), bounds[:,:,1] the smallest (rounded down).  Returns bounds."""
    c, b, dev, Hkv, _, d, _, _ = _paged(cache, block_table, kv_lens, q_start, _c_int(tokens, "tokens"))
    _call(dev, lib().lamp_kv_bounds, c, b, _bounds(bounds, dev, (cache.k.shape[0], Hkv, 2, d)))
    return bounds


def _tokens(q):
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q [T,Hq,d] expected")
    return q.shape[0]


def _queries(q, dev, d):
    """(pointer, token stride, head stride, heads) of q [T,Hq,d], checked."""
    if q.dtype is not _BF16 or q.get_device() != dev or q.stride(2) != 1:
        _must(q, "q", (_BF16,), dev)
    if q.shape[2] != d:
        raise ValueError("q of d = %d, a cache of %d" % (q.shape[2], d))
    return q.data_ptr(), q.stride(0), q.stride(1), q.shape[1]


@functools.lru_cache(maxsize=1024)
def _need(name, *sizes):
    """What a workspace size function of the library (of sizes alone) returns."""
    return int(getattr(lib(), name)(*sizes))


def _workspace(workspace, need, like, dev):
    """(pointer, bytes, the tensor) of a call's workspace: the caller's, or one of torch's of `need` bytes."""
    if workspace is None:
        if not need:
            return None, 0, None
        workspace = like.new_empty(need, dtype=torch.uint8)
        return workspace.data_ptr(), need, workspace
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the inputs' device")
    have = workspace.numel() * workspace.element_size()
    if not have and need:   # (its address is null)
        raise ValueError("workspace is empty")
    return workspace.data_ptr(), have, workspace


def _attn_out(q, out, dev):
    T, Hq, d = q.shape
    if out is None:
        return q.new_empty((T, Hq, d)), q.new_empty((T, Hq), dtype=_F32)
    o, lse = out
    _must(o, "o", (_BF16,), dev, (T, Hq, d))
    _must(lse, "lse", (_F32,), dev, (T, Hq))
    return o, lse


def select_pages_workspace_size(T, S, Hq, Hkv, d, width, budget):
    """Bytes of workspace one select_pages call needs (0: none)."""
    return int(lib().lamp_select_pages_workspace_size(T, S, Hq, Hkv, d, width, budget))


def select_pages(q, cache, bounds, block_table, kv_lens, budget, q_start=None, first=1, last=2, out=None, workspace=None):
    """For each new token and kv head the `budget` places of its sequence's block_table row whose pages could hold the
    largest logits: int32 [T,Hkv,budget], ascending, -1 behind the last.  q [T,Hq,d] as for attn_cache, bounds as
    kv_bounds keeps them.

    A page's score is an upper bound, over the heads that share the kv head, of q.k for its keys, with q rounded to 8
    bits: an exact number, so that the same places are selected everywhere (include/lamp.h).  The first `first` and the
    last `last` places in the token's sight are taken always; ties go to the lower place.  Rows of tokens behind
    q_start[S] are left as they are in `out`.  `workspace` as for attn_cache."""
    T = _tokens(q)
    c, b, dev, Hkv, _, d, S, width = _paged(cache, block_table, kv_lens, q_start, T)
    rows = _queries(q, dev, d)
    ranges = _bounds(bounds, dev, (cache.k.shape[0], Hkv, 2, d))
    budget, first, last = _c_int(budget, "budget"), _c_int(first, "first"), _c_int(last, "last")
    if budget <= 0:
        raise ValueError("budget must be positive")
    if out is None:
        out = kv_lens.new_empty((T, Hkv, budget))
    else:
        _must(out, "out", (_I32,), dev, (T, Hkv, budget))
    ws, size, keep = _workspace(workspace, _need("lamp_select_pages_workspace_size", T, S, rows[3], Hkv, d, width, budget), q, dev)
    _call(dev, lib().lamp_select_pages, *rows, c, b, ranges, budget, first, last, out.data_ptr(), ws, size)
    return out


def attn_pages_workspace_size(T, Hq, Hkv, d, page, budget):
    """Bytes of workspace one attn_pages call needs (0: none)."""
    return int(lib().lamp_attn_pages_workspace_size(T, Hq, Hkv, d, page, budget))


def attn_pages(q, cache, block_table, kv_lens, places, q_start=None, scale=None, out=None, workspace=None):
    """attn_cache (causal) where each new token and kv head sees only the keys of the places in its list: places int32
    [T,Hkv,budget], of select_pages or any others (one listed twice counts twice); what is not a place of the table holds
    no keys.
    Returns (o bf16 [T,Hq,d], lse fp32 [T,Hq])."""
    T = _tokens(q)
    c, b, dev, Hkv, page, d, _, _ = _paged(cache, block_table, kv_lens, q_start, T)
    rows = _queries(q, dev, d)
    if not isinstance(places, torch.Tensor) or places.dim() != 3 or places.shape[0] != T or places.shape[1] != Hkv \
            or places.shape[2] == 0:
        raise ValueError("places int32 [T,Hkv,budget] expected")
    if places.dtype is not _I32 or places.get_device() != dev or not places.is_contiguous():
        _must(places, "places", (_I32,), dev, places.shape)
    budget = places.shape[2]
    o, lse = _attn_out(q, out, dev)
    ws, size, keep = _workspace(workspace, _need("lamp_attn_pages_workspace_size", T, rows[3], Hkv, d, page, budget), q, dev)
    _call(dev, lib().lamp_attn_pages, *rows, c, b, places.data_ptr(), budget, d ** -0.5 if scale is None else float(scale),
          o.data_ptr(), lse.data_ptr(), ws, size)
    return o, lse


def attn_shared_workspace_size(T, S, groups, Hq, Hkv, d, page, width):
    """Bytes of workspace one attn_shared call needs."""
    return int(lib().lamp_attn_shared_workspace_size(T, S, groups, Hq, Hkv, d, page, width))


def attn_shared(q, cache, block_table, kv_lens, prefix_lens, group_start, q_start=None, scale=None, out=None,
                workspace=None):
    """attn_cache (causal) for sequences that share prefixes, each read once for all of its sequences: (o, lse).

    The sequences group_start[g] .. group_start[g+1]-1 (int32 [groups+1], from 0 to S) hold the same first prefix_lens[s]
    keys (int32 [S], the same for all of a group, rounded down to whole pages; 0: none), which all lie before their new
    tokens and are read through the table row of the group's first sequence.  The other arguments, and what comes out, as
    for attn_cache."""
    T = _tokens(q)
    c, b, dev, Hkv, page, d, S, width = _paged(cache, block_table, kv_lens, q_start, T)
    rows = _queries(q, dev, d)
    if not isinstance(group_start, torch.Tensor) or group_start.dim() != 1 or group_start.shape[0] < 2:
        raise ValueError("group_start int32 [groups + 1] expected")
    if not (prefix_lens.dtype is _I32 and group_start.dtype is _I32 and prefix_lens.get_device() == dev and group_start.get_device() == dev
            and prefix_lens.shape == (S,) and prefix_lens.is_contiguous() and group_start.is_contiguous()):
        _must(prefix_lens, "prefix_lens", (_I32,), dev, (S,))
        _must(group_start, "group_start", (_I32,), dev, group_start.shape)
    groups = group_start.shape[0] - 1
    o, lse = _attn_out(q, out, dev)
    ws, size, keep = _workspace(workspace, _need("lamp_attn_shared_workspace_size", T, S, groups, rows[3], Hkv, d, page, width), q, dev)
    _call(dev, lib().lamp_attn_shared, *rows, c, b, prefix_lens.data_ptr(), group_start.data_ptr(), groups,
          d ** -0.5 if scale is None else float(scale), o.data_ptr(), lse.data_ptr(), ws, size)
    return o, lse


def logits8(q, k, causal=True, window=0, row0=0, nrows=None, sr_seed=None):
    """e4m3 codes of the 8-bit logits of rows [row0, row0+nrows): uint8 [B,Hq,nrows,N], 0xFF invisible;
    with `sr_seed`, stochastically rounded (lamp_attn_logits8_sr)."""
    B, Hq, Hkv, N, d = _check_inputs(q, k)
    nrows = N - row0 if nrows is None else nrows
    y = torch.empty((B, Hq, nrows, N), dtype=torch.uint8, device=q.device)
    with torch.cuda.device(q.device):
        if sr_seed is None:
            rc = lib().lamp_attn_logits8(_ptr(q), _ptr(k), B, Hq, Hkv, N, d, int(causal), int(window), row0, nrows,
                                         _ptr(y), _stream(q.device))
        else:
            rc = lib().lamp_attn_logits8_sr(_ptr(q), _ptr(k), B, Hq, Hkv, N, d, int(causal), int(window), row0,
                                            nrows, int(sr_seed), _ptr(y), _stream(q.device))
    _check(rc)
    return y


def logits16(q, k, causal=True, window=0, row0=0, nrows=None):
    """e4m11 codes of the 16-bit logits: int16 bit patterns [B,Hq,nrows,N] (0xFFFF invisible)."""
    B, Hq, Hkv, N, d = _check_inputs(q, k)
    nrows = N - row0 if nrows is None else nrows
    y = torch.empty((B, Hq, nrows, N), dtype=torch.int16, device=q.device)
    with torch.cuda.device(q.device):
        rc = lib().lamp_attn_logits16(_ptr(q), _ptr(k), B, Hq, Hkv, N, d, int(causal), int(window), row0, nrows,
                                      _ptr(y), _stream(q.device))
    _check(rc)
    return y


def logits_sim(q, k, high, causal=True, window=0, row0=0, nrows=None):
    """SIM-profile logit values (high=False: 8-bit recursion, True: 16-bit):
    fp32 [B,Hq,nrows,N], NaN invisible."""
    B, Hq, Hkv, N, d = _check_inputs(q, k)
    nrows = N - row0 if nrows is None else nrows
    y = torch.empty((B, Hq, nrows, N), dtype=torch.float32, device=q.device)
    with torch.cuda.device(q.device):
        rc = lib().lamp_attn_logits_sim(_ptr(q), _ptr(k), B, Hq, Hkv, N, d, int(causal), int(window), row0, nrows,
                                        int(bool(high)), _ptr(y), _stream(q.device))
    _check(rc)
    return y


def selftest_e4m3(x):
    """(codes, raw codes) of fp32 CUDA tensor x by the device rounding sequence."""
    assert x.dtype == torch.float32 and x.is_cuda and x.is_contiguous()
    out = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    raw = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    with torch.cuda.device(x.device):
        _check(lib().lamp_selftest_e4m3(_ptr(x), _ptr(out), _ptr(raw), x.numel(), _stream(x.device)))
    return out, raw


def selftest_exp_doc(x):
    assert x.dtype == torch.float64 and x.is_cuda and x.is_contiguous()
    y = torch.empty_like(x)
    with torch.cuda.device(x.device):
        _check(lib().lamp_selftest_exp_doc(_ptr(x), _ptr(y), x.numel(), _stream(x.device)))
    return y


def get_tables(device=0):
    """(lut8 uint8[256], exp16 uint16[65536]) numpy copies of the device tables."""
    import numpy as np
    lut8 = np.empty(256, dtype=np.uint8)
    exp16 = np.empty(65536, dtype=np.uint16)
    _check(lib().lamp_get_tables(int(device), lut8.ctypes.data_as(ctypes.c_void_p),
                                 exp16.ctypes.data_as(ctypes.c_void_p)))
    return lut8, exp16


def get_exp16_parts(device=0):
    """uint32[65536]: the 16-bit exponentials as bf16 high (bits 15:0) and low
    (bits 31:16) parts."""
    import numpy as np
    parts = np.zeros(65536, dtype=np.uint32)
    _check(lib().lamp_get_exp16_parts(int(device), parts.ctypes.data_as(ctypes.c_void_p)))
    return parts


def get_sim_tables(device=0):
    """(sim8 uint16[112] bf16 bits, sim16 uint32[45056] FP32 patterns): the
    SIM profile's exponential tables, entry ((e - emin) << p) | m for the shift
    (2^p + m) 2^(e - p); p = 3, e in [-6, 7] and p = 11, e in [-14, 7]."""
    import numpy as np
    sim8 = np.zeros(112, dtype=np.uint16)
    sim16 = np.zeros(45056, dtype=np.uint32)
    _check(lib().lamp_get_sim_tables(int(device), sim8.ctypes.data_as(ctypes.c_void_p),
                                     sim16.ctypes.data_as(ctypes.c_void_p)))
    return sim8, sim16


def init(device=0):
    _check(lib().lamp_init(int(device)))


def shutdown():
    lib().lamp_shutdown()


def timing_enable(on=True):
    """Record HIP events around the prepass and forward kernel of each
    attn_fwd call (on the call's stream) until disabled."""
    _check(lib().lamp_timing_enable(1 if on else 0))


def timing_read():
    """(calls, forward-kernel ms summed, prepass ms summed) of the calls
    recorded since the previous read; waits for their events."""
    n, tf, tp = ctypes.c_int(0), ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(lib().lamp_timing_read(ctypes.byref(n), ctypes.byref(tf), ctypes.byref(tp)))
    return n.value, tf.value, tp.value


PHASE_NAMES = ("fused_pass", "emission", "barrier_B", "stage1", "exponentials", "barrier_E", "rescale_stage2",
               "pv_next_F0", "barrier_I", "prologue_epilogue")


def phase_read(reset=True):
    """Cycle sums per phase of the pipelined kernel and the wave count (a
    library built with the phase timer only; LampError otherwise)."""
    h = (ctypes.c_uint64 * (len(PHASE_NAMES) + 1))()
    _check(lib().lamp_phase_read(h, 1 if reset else 0))
    v = list(h)
    return dict(zip(PHASE_NAMES, v[:-1])), v[-1]


ISSUE_RATE_KINDS = ("fmac_f32", "fmac_f32_dpp", "cvt_pk_f32_fp8", "cvt_pk_fp8_f32", "emulated_step",
                    "emulated_step_sim")


def issue_rates():
    """Nanoseconds per wave-instruction per SIMD of the logit loops'
    instructions on the current device (dict keyed by ISSUE_RATE_KINDS;
    emulated_step is one step of the 8-bit loop, two multiply-adds per lane,
    emulated_step_sim one of the SIM profile's, one multiply-add)."""
    ns = (ctypes.c_double * len(ISSUE_RATE_KINDS))()
    _check(lib().lamp_issue_rates(ns, _stream(torch.device("cuda", torch.cuda.current_device()))))
    return dict(zip(ISSUE_RATE_KINDS, list(ns)))


def mask_stats(mask, nk):
    """Recompute statistics from a mask [B,Hq,nqb,ntiles*nk]: per key tile (nk
    sub-blocks, at least one active) the number of 16-bit sub-blocks, as a
    histogram 0..nk, plus counts per code.  Reporting only."""
    m = mask.reshape(-1, nk)
    active = (m != MASK_INACTIVE)
    tiles = active.any(dim=1)
    rec = ((m == MASK_STAGE1) | (m == MASK_STAGE2)).sum(dim=1)[tiles]
    hist = torch.bincount(rec.to(torch.int64), minlength=nk + 1).cpu().tolist()
    counts = torch.bincount(mask.reshape(-1).to(torch.int64), minlength=4).cpu().tolist()
    n_active = counts[0] + counts[1] + counts[2]
    return {
        "tile_hist": hist,
        "low": counts[0], "stage1": counts[1], "stage2": counts[2], "inactive": counts[3],
        "recompute_fraction": (counts[1] + counts[2]) / n_active if n_active else math.nan,
    }
