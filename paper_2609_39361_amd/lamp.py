"""Python binding of liblamp.so (the C ABI declared in include/lamp.h).

Argument marshalling only: every step of the forward pass runs in the HIP
kernels of the library.  PyTorch provides device memory and the stream.  The
library must have been built (python -m paper_2609_39361_amd.build); there is
no fallback path.
"""
import collections
import contextlib
import ctypes
import math
import os

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

class Rows(ctypes.Structure):
    """struct lamp_rows (include/lamp.h)."""
    _fields_ = [("p", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64),
                ("heads", ctypes.c_int)]


class _Cache(ctypes.Structure):
    """struct lamp_cache (include/lamp.h)."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("pages", ctypes.c_int), ("Hkv", ctypes.c_int), ("page", ctypes.c_int), ("d", ctypes.c_int)]


class _Batch(ctypes.Structure):
    """struct lamp_batch (include/lamp.h)."""
    _fields_ = [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("kv_lens", ctypes.c_void_p),
                ("q_start", ctypes.c_void_p), ("S", ctypes.c_int), ("T", ctypes.c_int), ("width", ctypes.c_int)]


# An 8-bit paged cache: codes k [pages,Hkv,page,d] and v [pages,Hkv,d,page] (float8_e4m3fn, V
# transposed within its page), scales k_scale and v_scale [pages,Hkv] (fp32 powers of two)
KVCache = collections.namedtuple("KVCache", "k v k_scale v_scale")

_FLOATS = (torch.bfloat16, torch.float32)


def kv_cache(pages, Hkv, d, page=64, device="cuda"):
    """An empty KVCache of `pages` pages of `page` tokens (zero codes and scales)."""
    z = dict(device=device)
    return KVCache(torch.zeros((pages, Hkv, page, d), dtype=torch.uint8, **z).view(torch.float8_e4m3fn),
                   torch.zeros((pages, Hkv, d, page), dtype=torch.uint8, **z).view(torch.float8_e4m3fn),
                   torch.zeros((pages, Hkv), dtype=torch.float32, **z), torch.zeros((pages, Hkv), dtype=torch.float32, **z))


def rope_table(n, rot, base=1e6, device="cuda"):
    """The rotation's table of positions 0 .. n-1: fp32 [n, rot], rot/2 cosines then rot/2 sines of
    position * base^(-2i/rot) (angles in fp64)."""
    inv = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    ang = torch.arange(n, dtype=torch.float64, device=device)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], dim=-1).float()


def _on(device):
    """The device made current, if it is not."""
    return contextlib.nullcontext() if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _check_tensor(t, name, dtypes, device, shape=None):
    """A CUDA tensor on `device` of one of `dtypes`, contiguous in its last dimension (`shape`: of that shape, dense)."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.device != device:
        raise ValueError("%s must be a %s tensor on %s" % (name, " or ".join(str(x) for x in dtypes), device))
    if shape is not None and (t.shape != shape or not t.is_contiguous()):
        raise ValueError("%s must be contiguous, of shape %s" % (name, tuple(shape)))
    if t.dim() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)


def _strides(t):
    """Strides in elements; 0 where only one index exists."""
    return tuple(s if n > 1 else 0 for s, n in zip(t.stride(), t.shape))


def _check_norm_rope(dev, d, gains, rope):
    for name, w in gains:
        if w is not None:
            _check_tensor(w, name, _FLOATS, dev, (d,))
    if rope is not None:
        _check_tensor(rope, "rope", (torch.float32,), dev)
        if rope.dim() != 2 or not rope.is_contiguous():
            raise ValueError("rope must be a contiguous [positions, rot] table")
    return (None, 0, 0) if rope is None else (rope.data_ptr(), rope.shape[0], rope.shape[1])


def qk_norm_rope(q, k=None, v=None, q_weight=None, k_weight=None, rope=None, positions=None, eps=1e-6, out=None):
    """RMS norm of every query and key head by the gains q_weight / k_weight [d] (None: not normed), then
    the rotation by `rope` (a table as of rope_table, None: not rotated), in one pass.

    Inputs bf16 or fp32 (all the same), outputs bf16; the last dimension contiguous, rows of 16-byte
    alignment (slices of a fused projection are fine).  Prompts: q [B,N,Hq,d], k and v [B,N,Hkv,d] give
    [B,H,N,d], what attn_fwd reads.  Tokens of a serving step: q [T,Hq,d], k and v [T,Hkv,d] give [T,H,d].
    `positions`: int32 [B,N] or [T]; default 0 .. N-1.  v is laid out (and rounded) with them.  `out`: the
    tensors to write into (None where the input is None), of the outputs' shapes with any strides; tokens
    may be written in place.  Returns (q, k, v), None for what was not given."""
    ins = (q, k, v)
    if not isinstance(q, torch.Tensor) or q.dim() not in (3, 4) or not q.is_cuda or q.dtype not in _FLOATS:
        raise ValueError("q must be a bf16 or fp32 CUDA tensor [B,N,Hq,d] or [T,Hq,d]")
    dev, prompt, d = q.device, q.dim() == 4, q.shape[-1]
    lead = q.shape[:-2]
    B, N = lead if prompt else (1, lead[0])
    for t, name in zip(ins, "qkv"):
        if t is not None:
            _check_tensor(t, name, (q.dtype,), dev)
            if t.dim() != q.dim() or t.shape[:-2] != lead or t.shape[-1] != d:
                raise ValueError("%s shape %s does not match q %s" % (name, tuple(t.shape), tuple(q.shape)))
    if k is not None and v is not None and k.shape != v.shape:
        raise ValueError("v shape %s differs from k %s" % (tuple(v.shape), tuple(k.shape)))
    table, npos, rot = _check_norm_rope(dev, d, (("q_weight", q_weight), ("k_weight", k_weight)), rope)
    if positions is not None:
        _check_tensor(positions, "positions", (torch.int32,), dev, lead)
    outs = []
    for i, t in enumerate(ins):
        o = None if out is None else out[i]
        shape = None if t is None else ((B, t.shape[2], N, d) if prompt else tuple(t.shape))
        if (t is None) != (o is None) and out is not None:
            raise ValueError("out must hold one tensor for each input")
        if o is not None:
            _check_tensor(o, "out[%d]" % i, (torch.bfloat16,), dev)
            if tuple(o.shape) != shape:
                raise ValueError("out[%d] must be of shape %s" % (i, shape))
        elif t is not None:
            o = torch.empty(shape, dtype=torch.bfloat16, device=dev)
        outs.append(o)
    if B * N and q.shape[-2]:
        ri, ro = (Rows * 3)(), (Rows * 3)()
        for i, (t, o) in enumerate(zip(ins, outs)):
            if t is not None:
                st, so = _strides(t), _strides(o)
                if prompt:
                    ri[i] = (t.data_ptr(), st[0], st[1], st[2], t.shape[2])
                    ro[i] = (o.data_ptr(), so[0], so[2], so[1], t.shape[2])
                else:
                    ri[i] = (t.data_ptr(), 0, st[0], st[1], t.shape[1])
                    ro[i] = (o.data_ptr(), 0, so[0], so[1], t.shape[1])
        f32 = torch.float32
        with _on(dev):
            _check(lib().lamp_qk_norm_rope(
                ri, ro, B, N, d, int(q.dtype == f32), None if q_weight is None else q_weight.data_ptr(),
                None if k_weight is None else k_weight.data_ptr(),
                int(q_weight is not None and q_weight.dtype == f32) + 2 * int(k_weight is not None and k_weight.dtype == f32),
                table, npos, rot, None if positions is None else positions.data_ptr(), float(eps), _stream(dev)))
    return tuple(outs)


def _paged(cache, block_table, kv_lens, q_start, T):
    """(lamp_cache, lamp_batch) of a call, checked."""
    kc, vc, ks, vs = cache
    if not isinstance(kc, torch.Tensor) or kc.dim() != 4 or not kc.is_cuda:
        raise ValueError("cache.k must be a float8_e4m3fn CUDA tensor [pages,Hkv,page,d]")
    dev = kc.device
    pages, Hkv, page, d = kc.shape
    fp8 = (torch.float8_e4m3fn,)
    _check_tensor(kc, "cache.k", fp8, dev, kc.shape)
    _check_tensor(vc, "cache.v", fp8, dev, (pages, Hkv, d, page))
    _check_tensor(ks, "cache.k_scale", (torch.float32,), dev, (pages, Hkv))
    _check_tensor(vs, "cache.v_scale", (torch.float32,), dev, (pages, Hkv))
    i32 = (torch.int32,)
    _check_tensor(block_table, "block_table", i32, dev)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [S, pages of a sequence]")
    S, width = block_table.shape
    _check_tensor(kv_lens, "kv_lens", i32, dev, (S,))
    if q_start is not None:
        _check_tensor(q_start, "q_start", i32, dev, (S + 1,))
    elif T != S:
        raise ValueError("without q_start there is one token for each of the %d sequences, not %d" % (S, T))
    c = _Cache(kc.data_ptr(), vc.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, Hkv, page, d)
    b = _Batch(block_table.data_ptr(), block_table.stride(0), kv_lens.data_ptr(),
               None if q_start is None else q_start.data_ptr(), S, T, width)
    return c, b, dev


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
    c, b, dev = _paged(cache, block_table, kv_lens, q_start, k.shape[0])
    _check_tensor(k, "k", _FLOATS, dev)
    _check_tensor(v, "v", (k.dtype,), dev)
    if k.shape[1:] != (c.Hkv, c.d):
        raise ValueError("k of %d heads and d = %d, a cache of %d and %d" % (k.shape[1], k.shape[2], c.Hkv, c.d))
    table, npos, rot = _check_norm_rope(dev, c.d, (("k_weight", k_weight),), rope)
    f32 = torch.float32
    with _on(dev):
        _check(lib().lamp_kv_append(
            k.data_ptr(), v.data_ptr(), int(k.dtype == f32), *_strides(k)[:2], *_strides(v)[:2],
            ctypes.byref(c), ctypes.byref(b), None if k_weight is None else k_weight.data_ptr(),
            int(k_weight is not None and k_weight.dtype == f32), table, npos, rot, float(eps), _stream(dev)))
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
    lse = -inf; tokens behind q_start[S] are left as they are in `out` = (o, lse).  `workspace`: a device
    tensor of attn_cache_workspace_size(...) bytes; by default one of torch's, on the current stream."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q [T,Hq,d] expected")
    T, Hq, d = q.shape
    c, b, dev = _paged(cache, block_table, kv_lens, q_start, T)
    _check_tensor(q, "q", (torch.bfloat16,), dev)
    if d != c.d:
        raise ValueError("q of d = %d, a cache of %d" % (d, c.d))
    if out is None:
        o = torch.empty((T, Hq, d), dtype=torch.bfloat16, device=dev)
        lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    else:
        o, lse = out
        _check_out(o, "o", (T, Hq, d), torch.bfloat16, dev)
        _check_out(lse, "lse", (T, Hq), torch.float32, dev)
    L = lib()
    if workspace is None:
        need = L.lamp_attn_cache_workspace_size(T, b.S, Hq, c.Hkv, d, c.page, b.width)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the inputs' device")
    with _on(dev):
        _check(L.lamp_attn_cache(
            q.data_ptr(), *_strides(q)[:2], Hq, ctypes.byref(c), ctypes.byref(b), int(causal), int(window),
            d ** -0.5 if scale is None else float(scale), o.data_ptr(), lse.data_ptr(),
            None if workspace is None else workspace.data_ptr(),
            0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(dev)))
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
