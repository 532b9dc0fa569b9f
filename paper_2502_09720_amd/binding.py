"""ctypes binding of libnestquant.so: argument marshalling only.

Device memory and streams come from torch; each function passes raw device pointers and
the current stream's handle to the matching C entry point and checks its status.
"""

import ctypes
import functools
import os
from typing import NamedTuple

PKG = os.path.dirname(os.path.abspath(__file__))
_LIB = None

NQ_OK, NQ_ERR_INVALID_ARG, NQ_ERR_UNSUPPORTED, NQ_ERR_HIP = 0, 1, 2, 3
NQ_F32, NQ_F16, NQ_BF16 = 0, 1, 2


class NQError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{message} (status {status})")
        self.status = status


class _Params(ctypes.Structure):
    _fields_ = [("q", ctypes.c_int32), ("k", ctypes.c_int32), ("base", ctypes.c_double),
                ("decoder", ctypes.c_int32), ("strategy", ctypes.c_int32),
                ("mult", ctypes.c_int32 * 4)]


class _KVCache(ctypes.Structure):
    _fields_ = [("k", _Params), ("v", _Params),
                *((n, ctypes.c_void_p) for n in ("k_codes", "k_beta", "k_scales", "v_codes",
                                                 "v_beta", "v_scales")),
                ("pages", ctypes.c_int64), ("heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("page", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _KVPrep(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("q_norm", ctypes.c_void_p),
                ("k_norm", ctypes.c_void_p), ("eps", ctypes.c_double),
                ("positions", ctypes.c_int64), ("rot", ctypes.c_int32),
                ("pairs", ctypes.c_int32), ("hadamard", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


DECODER_FULL = 0   # Alg. 2 with the Gosset oracle of Alg. 5
DECODER_M = 1      # NestQuantM (App. D): parity fixes at the first coordinate
FIRST_BETA = 0     # App. F: the smallest beta that does not overload
OPT_BETA = 1       # App. F: the beta of least reconstruction error


def library_path():
    return os.environ.get("NESTQUANT_LIB") or os.path.join(PKG, "libnestquant.so")


def library():
    """Load libnestquant.so (raises if it has not been built)."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it with `python -m paper_2502_09720_amd.build`")
        lib = ctypes.CDLL(path)
        vp, i64, u32p, f32p = ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p
        pp = ctypes.POINTER(_Params)
        lib.nq_encode.argtypes = [pp, vp, ctypes.c_int, i64, i64, i64, u32p, u32p, f32p, vp]
        lib.nq_rotate_encode.argtypes = lib.nq_encode.argtypes
        lib.nq_rotate_encode.restype = ctypes.c_int
        lib.nq_decode.argtypes = [pp, u32p, u32p, f32p, i64, i64, vp, ctypes.c_int, i64, vp]
        lib.nq_matmul.argtypes = [pp, u32p, u32p, f32p, i64, pp, u32p, u32p, f32p, i64, i64,
                                  f32p, i64, vp]
        lib.nq_matmul_ex.argtypes = [pp, u32p, u32p, f32p, i64, pp, u32p, u32p, f32p, i64, i64,
                                     f32p, i64, vp, i64, vp]
        lib.nq_matmul_stages.argtypes = [ctypes.c_int32, pp, u32p, u32p, f32p, i64, pp, u32p,
                                         u32p, f32p, i64, i64, f32p, i64, vp, i64, vp]
        lib.nq_encode_matmul.argtypes = [ctypes.c_int32, pp, vp, ctypes.c_int, i64, i64, i64,
                                         u32p, u32p, f32p, pp, u32p, u32p, f32p, i64, f32p, i64,
                                         vp, i64, vp]
        lib.nq_encode_matmul.restype = ctypes.c_int
        lib.nq_rotate.argtypes = [vp, ctypes.c_int, i64, i64, i64, f32p, i64, vp]
        lib.nq_rotate.restype = ctypes.c_int
        i32 = ctypes.c_int32
        lib.nq_beta_stats.argtypes = [i32, i32, vp, i64, ctypes.POINTER(ctypes.c_double), i32,
                                      vp, vp, vp]
        lib.nq_beta_stats.restype = ctypes.c_int
        lib.nq_beta_dp.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, i64, vp]
        lib.nq_beta_dp.restype = ctypes.c_int
        lib.nq_beta_dp_workspace_size.argtypes = [i64, i32]
        lib.nq_beta_dp_workspace_size.restype = i64
        lib.nq_matmul_workspace_size.argtypes = [i64, i64, i64]
        lib.nq_matmul_workspace_size.restype = i64
        kvp, hp = ctypes.POINTER(_KVCache), ctypes.POINTER(_Heads)
        lib.nq_kv_append.argtypes = [kvp, ctypes.POINTER(_KVPrep), i64, vp, vp, ctypes.c_int, hp,
                                     i32, hp, hp, hp, ctypes.c_int, vp]
        lib.nq_kv_append.restype = ctypes.c_int
        lib.nq_attend.argtypes = [kvp, vp, i64, vp, i64, vp, i64, i64, i64, i64, ctypes.c_double,
                                  ctypes.c_int, hp, i64, i32, hp, vp, vp, i64, vp]
        lib.nq_attend.restype = ctypes.c_int
        for f in (lib.nq_attend_workspace_size, lib.nq_attend_workspace_bound):
            f.argtypes = [i32, i32, i64, i32, i64, i64, i64, i64, i64]
            f.restype = i64
        for f in ("nq_encode", "nq_decode", "nq_matmul", "nq_matmul_ex", "nq_matmul_stages"):
            getattr(lib, f).restype = ctypes.c_int
        lib.nq_codes_words.argtypes = [i64, i64]
        lib.nq_codes_words.restype = i64
        lib.nq_beta_words.argtypes = [i64, i64]
        lib.nq_beta_words.restype = i64
        lib.nq_status_string.argtypes = [ctypes.c_int]
        lib.nq_status_string.restype = ctypes.c_char_p
        lib.nq_last_error.argtypes = []
        lib.nq_last_error.restype = ctypes.c_char_p
        lib.nq_version.argtypes = []
        lib.nq_version.restype = ctypes.c_int32
        _LIB = lib
    return _LIB


def _check(status):
    if status != NQ_OK:
        lib = library()
        raise NQError(status, lib.nq_last_error().decode() or lib.nq_status_string(status).decode())


def default_base(q, k):
    """beta_t = t * base with the k betas uniform on [0, 10] / q."""
    return 10.0 / (k * q)


@functools.lru_cache(maxsize=256)
def _params_of(q, k, base, decoder, strategy, mult):
    m = mult + (0,) * (4 - len(mult))
    return _Params(q, k, base, decoder, strategy, (ctypes.c_int32 * 4)(*m))


def _params(q, k, base, decoder=DECODER_FULL, strategy=FIRST_BETA, mult=None):
    """The nq_params of a call; the library only reads it, so equal ones are shared."""
    return _params_of(int(q), int(k), float(default_base(q, k) if base is None else base),
                      int(decoder), int(strategy),
                      () if mult is None else tuple(int(v) for v in mult))


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    # the handle alone: a Stream object of the current stream takes 2.8 us to make
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


@functools.lru_cache(maxsize=None)
def _dtype_codes():
    import torch
    return {torch.float32: NQ_F32, torch.float16: NQ_F16, torch.bfloat16: NQ_BF16}


def _dtype_code(dt):
    return _dtype_codes()[dt]


def nq_codes_words(rows, cols):
    return library().nq_codes_words(rows, cols)


def nq_beta_words(rows, cols):
    return library().nq_beta_words(rows, cols)


class Coded(NamedTuple):
    """A coded matrix: uint32 code words (stored in an int32 tensor), uint32 beta words,
    fp32 row scales, and the quantizer parameters (mult: the integer multiples of base that
    make the betas, None for 1..k)."""
    codes: "object"
    beta: "object"
    scales: "object"
    rows: int
    cols: int
    q: int
    k: int
    base: float
    decoder: int = DECODER_FULL
    mult: "object" = None


def encode(x, q=14, k=4, base=None, stream=None, out=None, decoder=DECODER_FULL,
           strategy=FIRST_BETA, mult=None, rotate=False):
    """nq_encode on a 2-D cuda tensor (fp32 / fp16 / bf16, unit stride along rows).
    ``decoder`` is the decoder the code is defined with (DECODER_FULL or DECODER_M);
    ``strategy`` picks the beta of each block (FIRST_BETA or OPT_BETA); ``mult`` gives the
    betas as integer multiples of base (k increasing integers in [1, 64]; None: 1..k).
    ``rotate``: the rows are Hadamard-rotated (as ``rotate``) before they are coded: in one
    pass (nq_rotate_encode) where the library supports it (First-beta; cols in 3584, 4096,
    7168, 8192, 14336, 16384), else as nq_rotate into a temporary fp32 matrix followed by
    nq_encode (same results)."""
    import torch
    if x.dim() != 2 or x.stride(1) != 1 or not x.is_cuda:
        raise ValueError("x must be a 2-D cuda tensor with unit column stride")
    rows, cols = x.shape
    lib = library()
    if cols < 8 or cols % 8:
        raise ValueError("cols must be a positive multiple of 8")
    if out is None:
        nw, bw = lib.nq_codes_words(rows, cols), lib.nq_beta_words(rows, cols)
        codes = torch.empty(nw, dtype=torch.int32, device=x.device)
        beta = torch.empty(bw, dtype=torch.int32, device=x.device)
        scales = torch.empty(rows, dtype=torch.float32, device=x.device)
    else:
        codes, beta, scales = out
    p = _params(q, k, base, decoder, strategy, mult)

    def call(fn, src):
        return fn(ctypes.byref(p), src.data_ptr(), _dtype_code(src.dtype), rows,
                  cols, src.stride(0), codes.data_ptr(),
                  beta.data_ptr(), scales.data_ptr(),
                  _stream(stream))
    st = call(lib.nq_rotate_encode if rotate else lib.nq_encode, x)
    if rotate and st == NQ_ERR_UNSUPPORTED:
        st = call(lib.nq_encode, _rotated(x, stream))                     # two passes
    _check(st)
    return Coded(codes, beta, scales, rows, cols, int(q), int(k), p.base, int(decoder),
                 None if mult is None else tuple(int(v) for v in mult))


def decode(coded, out_dtype=None, stream=None, out=None):
    """nq_decode: the reconstruction r * beta_t * p as a rows x cols tensor."""
    import torch
    dt = torch.float32 if out_dtype is None else out_dtype
    if out is None:
        out = torch.empty(coded.rows, coded.cols, dtype=dt, device=coded.codes.device)
    p = _params(coded.q, coded.k, coded.base, coded.decoder, mult=coded.mult)
    lib = library()
    _check(lib.nq_decode(ctypes.byref(p), coded.codes.data_ptr(),
                         coded.beta.data_ptr(),
                         coded.scales.data_ptr(), coded.rows, coded.cols,
                         out.data_ptr(), _dtype_code(out.dtype), out.stride(0),
                         _stream(stream)))
    return out


STAGE_DECODE = 1
STAGE_CONTRACT = 2
CONTRACT_INT8 = 4
ROTATE_A = 8


def matmul(a, w, stream=None, out=None, workspace=None, stages=STAGE_DECODE | STAGE_CONTRACT,
           int8=False):
    """nq_matmul: C = A_hat W_hat^T (fp32, M x N) from two coded operands.

    The decode-once workspace is taken from torch's allocator unless given.  ``stages``
    selects part of the call (nq_matmul_stages): STAGE_DECODE fills the workspace,
    STAGE_CONTRACT computes C from it; both (the default) is the whole product.  ``int8``
    insists on exact int8 tiles and int8 matrix cores (needs k * q <= 63); without it the
    library takes them by itself where every tile value fits."""
    import torch
    if a.cols != w.cols:
        raise ValueError("K mismatch")
    if out is None:
        out = torch.empty(a.rows, w.rows, dtype=torch.float32, device=a.codes.device)
    pa = _params(a.q, a.k, a.base, a.decoder, mult=a.mult)
    pw = _params(w.q, w.k, w.base, w.decoder, mult=w.mult)
    lib = library()
    need = lib.nq_matmul_workspace_size(a.rows, w.rows, a.cols)
    if need < 0:
        raise ValueError("invalid matmul shape")
    whole = stages == STAGE_DECODE | STAGE_CONTRACT
    if need > 0 and (workspace is None or workspace.numel() * workspace.element_size() < need):
        if not whole:
            raise ValueError("a staged matmul needs a workspace of matmul_workspace_size bytes")
        workspace = torch.empty(need, dtype=torch.uint8, device=a.codes.device)
        if stream is not None:
            workspace.record_stream(stream)       # freed on return, in use on `stream`
    ws_ptr = workspace.data_ptr() if need > 0 else 0
    args = (ctypes.byref(pa), a.codes.data_ptr(),
            a.beta.data_ptr(), a.scales.data_ptr(), a.rows,
            ctypes.byref(pw), w.codes.data_ptr(),
            w.beta.data_ptr(), w.scales.data_ptr(), w.rows,
            a.cols, out.data_ptr(), out.stride(0), ws_ptr,
            need, _stream(stream))
    if whole and not int8:
        _check(lib.nq_matmul_ex(*args))
    else:
        _check(lib.nq_matmul_stages(stages | (CONTRACT_INT8 if int8 else 0), *args))
    return out


def matmul_direct(a, w, stream=None, out=None):
    """nq_matmul: C = A_hat W_hat^T with no workspace (each workgroup decodes the code words
    of its own rows into on-chip memory); the same product as ``matmul``."""
    import torch
    if a.cols != w.cols:
        raise ValueError("K mismatch")
    if out is None:
        out = torch.empty(a.rows, w.rows, dtype=torch.float32, device=a.codes.device)
    pa = _params(a.q, a.k, a.base, a.decoder, mult=a.mult)
    pw = _params(w.q, w.k, w.base, w.decoder, mult=w.mult)
    _check(library().nq_matmul(
        ctypes.byref(pa), a.codes.data_ptr(), a.beta.data_ptr(),
        a.scales.data_ptr(), a.rows, ctypes.byref(pw),
        w.codes.data_ptr(), w.beta.data_ptr(),
        w.scales.data_ptr(), w.rows, a.cols, out.data_ptr(),
        out.stride(0), _stream(stream)))
    return out


def encode_matmul(x, w, q=14, k=4, base=None, decoder=DECODER_FULL, strategy=FIRST_BETA,
                  mult=None, stream=None, out=None, coded_out=None, workspace=None,
                  int8=False, rotate=False):
    """nq_encode_matmul: codes the activation x (2-D cuda tensor, as ``encode``) and returns
    (its Coded operand, C = A_hat W_hat^T) from one call, the encoder writing A's decoded
    tiles straight into the product's workspace.  The same results as ``encode`` then
    ``matmul``.  ``rotate``: x's rows are Hadamard-rotated before they are coded (w must hold
    the codes of rotated weight rows): NQ_ROTATE_A where the library supports it (as for
    ``encode``), else nq_rotate into a temporary fp32 matrix first (same results)."""
    import torch
    if x.dim() != 2 or x.stride(1) != 1 or not x.is_cuda:
        raise ValueError("x must be a 2-D cuda tensor with unit column stride")
    M, K = x.shape
    if K != w.cols:
        raise ValueError("K mismatch")
    lib = library()
    if coded_out is None:
        codes = torch.empty(max(lib.nq_codes_words(M, K), 0), dtype=torch.int32, device=x.device)
        beta = torch.empty(max(lib.nq_beta_words(M, K), 0), dtype=torch.int32, device=x.device)
        scales = torch.empty(M, dtype=torch.float32, device=x.device)
    else:
        codes, beta, scales = coded_out
    if out is None:
        out = torch.empty(M, w.rows, dtype=torch.float32, device=x.device)
    need = lib.nq_matmul_workspace_size(M, w.rows, K)
    if need < 0:
        raise ValueError("invalid matmul shape")
    if need > 0 and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        if stream is not None:
            workspace.record_stream(stream)       # freed on return, in use on `stream`
    pa = _params(q, k, base, decoder, strategy, mult)
    pw = _params(w.q, w.k, w.base, w.decoder, mult=w.mult)

    def call(flags, src):
        return lib.nq_encode_matmul(
            flags, ctypes.byref(pa), src.data_ptr(), _dtype_code(src.dtype), M,
            K, src.stride(0), codes.data_ptr(),
            beta.data_ptr(), scales.data_ptr(),
            ctypes.byref(pw), w.codes.data_ptr(),
            w.beta.data_ptr(), w.scales.data_ptr(), w.rows,
            out.data_ptr(), out.stride(0),
            workspace.data_ptr() if need > 0 else 0, need, _stream(stream))
    flags = CONTRACT_INT8 if int8 else 0
    st = call(flags | (ROTATE_A if rotate else 0), x)
    if rotate and st == NQ_ERR_UNSUPPORTED:
        st = call(flags, _rotated(x, stream))                                # two passes
    _check(st)
    a = Coded(codes, beta, scales, M, K, int(q), int(k), pa.base, int(decoder),
              None if mult is None else tuple(int(v) for v in mult))
    return a, out


def rotate(x, out=None, stream=None):
    """nq_rotate: y = x U in fp32 for every row of a 2-D cuda tensor (Sec. 5 Hadamard
    rotation; cols = 2^k or 28 * 2^k, at most 32768)."""
    import torch
    if x.dim() != 2 or x.stride(1) != 1 or not x.is_cuda:
        raise ValueError("x must be a 2-D cuda tensor with unit column stride")
    rows, cols = x.shape
    if out is None:
        out = torch.empty(rows, cols, dtype=torch.float32, device=x.device)
    _check(library().nq_rotate(x.data_ptr(), _dtype_code(x.dtype), rows, cols,
                               x.stride(0), out.data_ptr(), out.stride(0),
                               _stream(stream)))
    return out


def _rotated(x, stream):
    """nq_rotate of x into a new fp32 matrix (the two-pass form of the rotating calls).  The
    temporary is freed when the caller returns, so it is marked as in use on `stream` until
    the work queued there is done."""
    y = rotate(x, stream=stream)
    if stream is not None:
        y.record_stream(stream)
    return y


def matmul_workspace_size(M, N, K):
    return library().nq_matmul_workspace_size(M, N, K)


def beta_stats(v, betas, q, decoder=DECODER_FULL, stream=None):
    """nq_beta_stats: for sample 8-vectors v (n x 8 fp32 cuda tensor) and the increasing
    candidate betas (a sequence of at most 64 floats), the squared coding error mse (n x m
    fp64) and the overload flags (n x m uint8) of every sample at every beta."""
    import torch
    if v.dim() != 2 or v.shape[1] != 8 or v.dtype != torch.float32 or not v.is_contiguous():
        raise ValueError("v must be a contiguous n x 8 float32 cuda tensor")
    n, m = v.shape[0], len(betas)
    mse = torch.empty(n, m, dtype=torch.float64, device=v.device)
    over = torch.empty(n, m, dtype=torch.uint8, device=v.device)
    b = (ctypes.c_double * m)(*[float(x) for x in betas])
    _check(library().nq_beta_stats(int(q), int(decoder), v.data_ptr(), n, b,
                                   m, mse.data_ptr(),
                                   over.data_ptr(), _stream(stream)))
    return mse, over


def beta_dp(mse, over, k, stream=None, workspace=None):
    """nq_beta_dp (Alg. 6): the k grid indices (int32 cuda tensor, increasing; -1 if every
    beta overloads) minimizing the First-beta error, and that error (fp64 cuda scalar).  The
    scratch memory (nq_beta_dp_workspace_size bytes) comes from torch's allocator unless
    given."""
    import torch
    n, m = mse.shape
    lib = library()
    chosen = torch.empty(k, dtype=torch.int32, device=mse.device)
    loss = torch.empty((), dtype=torch.float64, device=mse.device)
    need = lib.nq_beta_dp_workspace_size(n, m)
    if need < 0:
        raise ValueError("invalid beta_dp shape")
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=mse.device)
        if stream is not None:
            workspace.record_stream(stream)       # freed on return, in use on `stream`
    _check(lib.nq_beta_dp(mse.data_ptr(), over.data_ptr(),
                          n, m, int(k), chosen.data_ptr(),
                          loss.data_ptr(), workspace.data_ptr(),
                          workspace.numel() * workspace.element_size(), _stream(stream)))
    return chosen, loss


# ----------------------------------------------------------------------------------------
# a coded KV cache
# ----------------------------------------------------------------------------------------

_PAIRS = {"halves": 0, "neighbours": 1}


class KVCache:
    """Pages of coded keys and values (made by ``kv_cache``): ``k`` and ``v`` are the two pools as
    coded matrices of pages * heads * page rows of dim entries, slot s of head h in page p at
    row (p * heads + h) * page + s (``decode`` reads them)."""

    __slots__ = ("k", "v", "pages", "heads", "dim", "page", "_c", "_device")

    def __init__(self, k, v, pages, heads, dim, page):
        self.k, self.v = k, v
        self.pages, self.heads, self.dim, self.page = pages, heads, dim, page
        ps = [_params(c.q, c.k, c.base, c.decoder, mult=c.mult) for c in (k, v)]
        self._c = _KVCache(*ps, *(t.data_ptr() for c in (k, v) for t in (c.codes, c.beta, c.scales)),
                           pages, heads, dim, page, 0)
        self._device = k.codes.get_device()       # its index, -1: not on a GPU


def kv_cache(pages=None, heads=8, dim=128, page=64, q=14, k=4, base=None, decoder=DECODER_FULL,
             mult=None, values=None, pools=None, device="cuda"):
    """A coded KV cache of ``pages`` pages of ``page`` tokens (16, 32, 64, 128 or 256) of
    ``heads`` heads of ``dim`` entries (64, 128 or 256).  q, k, base, decoder and mult are the
    quantizer's parameters (as ``encode``) for the keys and, unless ``values`` (a dict of the
    same) says otherwise, the values; ``attend`` needs one decoder for both.  ``pools``: the six
    arrays (codes, beta words and scales of the keys, then of the values) of the caller,
    contiguous, instead of new ones, whose scales are zero; the cache then has as many pages as
    they hold."""
    import torch
    if dim < 8 or dim % 8 or heads < 1 or page < 1:
        raise ValueError("invalid cache shape")
    nb, nw = dim // 8, (dim + 127) // 128
    if pools is None:
        if pages is None or pages < 0:
            raise ValueError("pages is missing")
        rows = pages * heads * page
        pools = [torch.empty(rows * n, dtype=torch.int32, device=device) if n else
                 torch.zeros(rows, dtype=torch.float32, device=device) for n in (nb, nw, 0)] + [
                 torch.empty(rows * n, dtype=torch.int32, device=device) if n else
                 torch.zeros(rows, dtype=torch.float32, device=device) for n in (nb, nw, 0)]
    else:
        rows = pools[2].numel()
        if rows % (heads * page) or (pages is not None and rows != pages * heads * page):
            raise ValueError("the pools do not hold whole pages")
        pages = rows // (heads * page)
        for t, n in zip(pools, (nb, nw, 1, nb, nw, 1)):
            if t.numel() != rows * n or not t.is_contiguous() or t.element_size() != 4:
                raise ValueError("pools must be contiguous 32-bit arrays of the cache's sizes")
            if t.device != pools[0].device:
                raise ValueError("pools must be on one device")
        for t in (pools[2], pools[5]):
            if t.dtype != torch.float32:
                raise ValueError("scales must be float32")
    own = dict(q=q, k=k, base=base, decoder=decoder, mult=mult)
    coded = []
    for o, arrays in ((own, pools[:3]), ({**own, **(values or {})}, pools[3:])):
        p = _params(o["q"], o["k"], o["base"], o["decoder"], mult=o["mult"])
        coded.append(Coded(*arrays, rows, dim, int(o["q"]), int(o["k"]), p.base, int(o["decoder"]),
                           None if o["mult"] is None else tuple(int(m) for m in o["mult"])))
    return KVCache(*coded, pages, heads, dim, page)


def _heads(x, name, device):
    """A tokens x heads x dim tensor as the library takes it."""
    s = x.stride()
    if len(s) != 3 or s[2] != 1 or x.get_device() != device:
        raise ValueError(f"{name} must be a tokens x heads x dim tensor with unit last stride on the "
                         "cache's GPU")
    if (s[0] | s[1]) & 7:       # the stride of a single token or head steps nowhere, whatever it is
        s = [0 if n == 1 else step for n, step in zip(x.shape, s)]
    return _Heads(x.data_ptr(), s[0], s[1])


def _index(x, n, dtype, name, device):
    if x.dtype != dtype or x.numel() != n or not x.is_contiguous() or x.get_device() != device:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} entries on the cache's GPU")
    return x.data_ptr()


def _empty(shape, dtype, device, stream):
    """Memory for a call on ``stream``: from that stream's own pool, so that what is still to run on
    the current stream with memory it freed is not written over, and memory freed while the call
    runs is handed out again behind it."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def kv_append(cache, q, k, v, slots, positions=None, cos=None, sin=None, pairs="halves",
              q_norm=None, k_norm=None, eps=1e-5, hadamard=True, out=None, stream=None):
    """nq_kv_append: codes the keys and values of new tokens (tokens x heads x dim cuda tensors
    of one type, any strides with unit last) into their slots (int64, one a token: page * page
    size + slot in the page; -1 leaves a token out) and returns the queries (tokens x
    query heads x dim, or None) as attention takes them.

    Queries and keys are normed (``q_norm``, ``k_norm``: dim float32 weights), rotated by
    position (``cos``, ``sin``: positions x rot / 2 float32 tables, ``positions`` int32, one a
    token, not read without tables; ``pairs``: "halves" or "neighbours") and, with ``hadamard``,
    by H / sqrt(dim); keys and values are coded as ``encode`` codes rows.  ``out`` may have another
    type than q.  With ``stream``, a new output belongs to that stream's memory."""
    import torch
    device = cache._device
    if device < 0:
        raise ValueError("the cache's pools are not on a GPU")
    tokens, heads, dim = k.shape
    if heads != cache.heads or dim != cache.dim or v.shape != k.shape:
        raise ValueError("k and v must be tokens x heads x dim of the cache")
    if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise ValueError("q, k and v must have one type")
    rot = rows = 0
    if cos is not None or sin is not None:
        if cos is None or sin is None or positions is None:
            raise ValueError("cos, sin and positions go together")
        for t in (cos, sin):
            if t.dim() != 2 or t.dtype != torch.float32 or not t.is_contiguous() or t.get_device() != device:
                raise ValueError("cos and sin must be contiguous 2-D float32 tensors on the cache's GPU")
        if sin.shape != cos.shape:
            raise ValueError("cos and sin differ in shape")
        rows, rot = cos.shape
        rot *= 2
    for t, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        if t is not None:
            _index(t, dim, torch.float32, name, device)
    prep = _KVPrep(cos.data_ptr() if rot else None, sin.data_ptr() if rot else None,
                   None if q_norm is None else q_norm.data_ptr(),
                   None if k_norm is None else k_norm.data_ptr(), float(eps), rows, rot,
                   _PAIRS[pairs], 1 if hadamard else 0, 0)
    hq = ho = None
    q_heads = 0
    if q is not None:
        if q.shape[0] != tokens or q.shape[2] != dim:
            raise ValueError("q must be tokens x query heads x dim")
        q_heads = q.shape[1]
        if out is None:
            out = _empty((tokens, q_heads, dim), q.dtype, q.device, stream)
        elif out.shape != q.shape:
            raise ValueError("out must have q's shape")
        hq, ho = _heads(q, "q", device), _heads(out, "out", device)
    _check(library().nq_kv_append(
        cache._c, prep, tokens, _index(slots, tokens, torch.int64, "slots", device),
        _index(positions, tokens, torch.int32, "positions", device) if rot else None, _dtype_code(k.dtype),
        hq, q_heads, _heads(k, "k", device), _heads(v, "v", device), ho,
        _dtype_code(out.dtype) if q is not None else NQ_F32, _stream(stream)))
    return out if q is not None else None


def attend_workspace_size(cache, tokens, q_heads, seqs, max_queries=1, max_length=1, window=0,
                          sinks=0):
    """Scratch bytes that serve every ``attend`` of at most these sizes, and of this window or a
    smaller one (nq_attend_workspace_bound): a workspace to keep."""
    n = library().nq_attend_workspace_bound(cache.heads, cache.dim, tokens, q_heads, seqs,
                                            min(max_queries, tokens), max_length, window, sinks)
    if n < 0:
        raise ValueError("invalid attend shape")
    return n


def attend(cache, q, table, lengths, starts=None, max_queries=None, max_length=None, window=0,
           sinks=0, scale=None, out=None, lse=None, workspace=None, stream=None):
    """nq_attend: attention of the queries q (tokens x query heads x dim) over a coded cache.

    ``table`` (int32, sequences x pages) names each sequence's pages, ``lengths`` (int32) its
    tokens in the cache, ``starts`` (int32, sequences + 1; None: one query a sequence) its
    rows of q, the last of them at the sequence's last position.  A query sees the tokens up to
    its position, with ``window`` > 0 the last ``window`` of them and the first ``sinks``.
    ``max_queries`` and ``max_length`` bound the queries and the tokens of a sequence (None: as
    many as q and the table allow, at the cost of scratch memory and of idle workgroups).
    ``workspace``: scratch memory of ``attend_workspace_size`` bytes (a call with less, or None,
    takes its own from torch's allocator).
    Returns out (q's shape and type); ``lse`` (tokens x query heads float32), if given,
    receives the logarithms of the softmax sums."""
    import torch
    device = cache._device
    if device < 0:
        raise ValueError("the cache's pools are not on a GPU")
    tokens, q_heads, dim = q.shape
    if dim != cache.dim:
        raise ValueError("q must be tokens x query heads x dim of the cache")
    seqs = lengths.numel()
    ok = table.dim() == 2 and table.dtype == torch.int32 and table.get_device() == device
    if ok:
        (rows, pages), (step, unit) = table.shape, table.stride()
    if not ok or rows != seqs or (pages > 0 and unit != 1):
        raise ValueError("table must be a sequences x pages int32 tensor with unit last stride on the "
                         "cache's GPU")
    if starts is None:
        if tokens != seqs:
            raise ValueError("without starts there is one query a sequence")
        max_queries = 1
    elif max_queries is None or max_queries > tokens:
        max_queries = tokens
    if seqs == 1 or step < pages:
        step = pages
        if seqs > 1:                     # rows that overlap, as an expanded row's
            with torch.cuda.stream(stream):
                table = table.contiguous()
    most = pages * cache.page
    if max_length is None:
        max_length = most
    elif max_length > most:
        raise ValueError("max_length exceeds the table's pages")
    if out is None:
        out = _empty((tokens, q_heads, dim), q.dtype, q.device, stream)
    elif out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out must have q's shape and type")
    if lse is not None:
        _index(lse, tokens * q_heads, torch.float32, "lse", device)
    if workspace is not None and (workspace.get_device() != device or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous tensor on the cache's GPU")
    lib = library()
    need = lib.nq_attend_workspace_size(cache.heads, dim, tokens, q_heads, seqs, max_queries,
                                        max_length, window, sinks)
    if need < 0:
        raise ValueError("invalid attend shape")
    if need > 0 and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _empty((need,), torch.uint8, q.device, stream)
    _check(lib.nq_attend(
        cache._c, table.data_ptr(), max(step, 1),
        _index(lengths, seqs, torch.int32, "lengths", device), seqs,
        None if starts is None else _index(starts, seqs + 1, torch.int32, "starts", device), max_queries,
        max_length, window, sinks, dim ** -0.5 if scale is None else scale, _dtype_code(q.dtype),
        _heads(q, "q", device), tokens, q_heads, _heads(out, "out", device), None if lse is None else lse.data_ptr(),
        workspace.data_ptr() if need > 0 else None, need, _stream(stream)))
    return out
