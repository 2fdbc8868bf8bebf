"""ELSAA attention operator on AMD Instinct MI355X (gfx950).

Thin Python binding of the C-ABI library ``libelsaa.so`` (declared in
``include/elsaa.h``).  The functions below only marshal arguments: they
allocate the output, ``saved`` and ``workspace`` buffers with torch on the
tensors' device, pass raw device pointers and torch's current HIP stream,
and raise if the library reports an error.  Every step of the operator runs
in the library's HIP kernels; there is no other code path.  If the library
has not been built, importing works but every call raises.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libelsaa.so")
_lib = None

F32, BF16, I8 = 0, 1, 2
_STATUS = {0: "ok", -1: "invalid argument", -2: "unsupported", -3: "buffer too small", -4: "HIP error"}


class ElsaaError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"elsaa error {status} ({_STATUS.get(status, '?')}): {msg}")
        self.status = status


class _Config(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("N", C.c_int32), ("d_h", C.c_int32),
                ("k", C.c_int32), ("r", C.c_int32), ("race_bits", C.c_int32),
                ("sort_bits", C.c_int32), ("n0", C.c_int32), ("causal", C.c_int32),
                ("dtype", C.c_int32), ("beta", C.c_float), ("lam", C.c_float),
                ("eps", C.c_float), ("scale", C.c_float), ("neighbors", C.c_int32),
                ("m_one", C.c_int32)]


class _SavedLayout(C.Structure):
    _fields_ = [("perm_q", C.c_size_t), ("perm_k", C.c_size_t), ("m", C.c_size_t),
                ("o_sparse", C.c_size_t), ("o_lowrank", C.c_size_t), ("u_q", C.c_size_t),
                ("u_k", C.c_size_t), ("race_states", C.c_size_t), ("total", C.c_size_t)]


class _TokenRules(C.Structure):
    _fields_ = [("gate_hidden", C.c_int32), ("W1", C.c_void_p), ("b1", C.c_void_p), ("W2", C.c_void_p),
                ("b2", C.c_void_p), ("lambda_rule", C.c_int32), ("lam_w", C.c_void_p),
                ("lam_b", C.c_void_p), ("lam_c", C.c_void_p), ("lambda_min", C.c_float)]


class _GemmDesc(C.Structure):
    _fields_ = [("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("trans_a", C.c_int32),
                ("trans_b", C.c_int32), ("lda", C.c_int64), ("ldb", C.c_int64), ("ldc", C.c_int64),
                ("a_heads", C.c_int32), ("b_heads", C.c_int32), ("c_heads", C.c_int32),
                ("seq", C.c_int32), ("c_dtype", C.c_int32)]


class _NormDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("dtype", C.c_int32), ("y_dtype", C.c_int32),
                ("eps", C.c_float), ("ldx", C.c_int64), ("ldr", C.c_int64), ("lds", C.c_int64),
                ("ldy", C.c_int64)]


class _QuantDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("dtype", C.c_int32), ("ld", C.c_int64),
                ("ldq", C.c_int64), ("heads", C.c_int32), ("seq", C.c_int32)]


class _GemmI8Desc(C.Structure):
    _fields_ = [("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("lda", C.c_int64), ("ldb", C.c_int64),
                ("ldc", C.c_int64), ("c_heads", C.c_int32), ("seq", C.c_int32), ("c_dtype", C.c_int32)]


class _DecayDesc(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("N", C.c_int32), ("d_h", C.c_int32), ("dtype", C.c_int32),
                ("scale", C.c_float)] + [(n + "_batch", C.c_int64) for n in ("q", "k", "v", "o", "dq", "dk", "dv")] + [
                    ("zero_tail", C.c_int32)]


@dataclasses.dataclass
class Config:
    """Operator settings (names follow the paper; see include/elsaa.h)."""
    B: int
    H: int
    N: int
    d_h: int
    k: int                  # sortLSH block size b
    r: int                  # RACE features L * 2^race_bits
    causal: bool
    dtype: str = "bf16"     # storage dtype of Q, K, V, O, dO, dQ, dK, dV
    race_bits: int = 4
    sort_bits: int = 5
    n0: int = 0             # <= 0 -> 2k
    beta: float = 1.0
    lam: float = 1.0
    eps: float = 1e-6
    scale: float = 0.0      # <= 0 -> 1/sqrt(d_h)
    neighbors: int = 0      # neighbouring sorted blocks seen on each side
    m_one: bool = False     # m_sparse = 1 (the Sort_Lsh_RACE ablation)

    def c(self) -> _Config:
        return _Config(self.B, self.H, self.N, self.d_h, self.k, self.r, self.race_bits,
                       self.sort_bits, self.n0, int(self.causal),
                       BF16 if self.dtype == "bf16" else F32, self.beta, self.lam, self.eps,
                       self.scale, self.neighbors, int(self.m_one))

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32


def load():
    """Load libelsaa.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ElsaaError(-4, f"{LIB_PATH} not built; run paper_2607_20214_amd/build.py")
        lib = C.CDLL(LIB_PATH)
        P, S = C.c_void_p, C.c_size_t
        lib.elsaa_num_levels.argtypes = [P]
        lib.elsaa_perm_length.argtypes = [P]
        lib.elsaa_perm_length.restype = C.c_int64
        lib.elsaa_saved_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
        lib.elsaa_workspace_bytes.argtypes = [P, C.c_int, C.POINTER(C.c_size_t)]
        lib.elsaa_get_saved_layout.argtypes = [P, P]
        lib.elsaa_select.argtypes = [P, P, P, P, P, P, P, S, P]
        lib.elsaa_select_noalloc.argtypes = [P, P, P, P, P, P, P]
        lib.elsaa_fwd.argtypes = [P, P, P, P, P, P, P, P, P, P, P, P, S, P, S, P]
        lib.elsaa_bwd.argtypes = [P, P, P, P, P, P, P, P, P, P, P, P, S, P, P, P, P, P, P, S, P]
        lib.elsaa_gemm_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
        lib.elsaa_gemm.argtypes = [P, P, P, P, P, S, P]
        lib.elsaa_token_rules_fwd.argtypes = [P, P, P, P, P, P]
        lib.elsaa_token_rules_workspace_bytes.argtypes = [P, P, C.POINTER(C.c_size_t)]
        lib.elsaa_token_rules_bwd.argtypes = [P, P, P, P, P, P] + [P] * 7 + [P, S, P]
        lib.elsaa_rms_norm_fwd.argtypes = [P, P, P, P, P, P, P, P]
        lib.elsaa_rms_norm_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
        lib.elsaa_rms_norm_bwd.argtypes = [P, P, P, P, P, P, P, P, S, P]
        lib.elsaa_quantize_rows.argtypes = [P, P, P, P, P]
        lib.elsaa_gemm_i8_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
        lib.elsaa_gemm_i8.argtypes = [P, P, P, P, P, P, P, S, P]
        lib.elsaa_decay_workspace_bytes.argtypes = [P, C.c_int, C.POINTER(C.c_size_t)]
        lib.elsaa_decay_fwd.argtypes = [P] * 10 + [S, P]
        lib.elsaa_decay_bwd.argtypes = [P] * 14 + [S, P]
        lib.elsaa_decay_step.argtypes = [P] * 9
        lib.elsaa_profile_enable.argtypes = [C.c_int]
        lib.elsaa_profile_count.argtypes = []
        lib.elsaa_profile_get.argtypes = [C.c_int, C.c_char_p, S, C.POINTER(C.c_double),
                                          C.POINTER(C.c_int64)]
        lib.elsaa_status_string.restype = C.c_char_p
        lib.elsaa_status_string.argtypes = [C.c_int]
        lib.elsaa_last_error.restype = C.c_char_p
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != 0:
        raise ElsaaError(rc, load().elsaa_last_error().decode())


def _p(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(dev) -> C.c_void_p:
    return C.c_void_p(torch.cuda.current_stream(dev).cuda_stream)


def profile_enable(on: bool = True):
    """Start (clearing old totals) or stop per-kernel event timing in the library."""
    _check(load().elsaa_profile_enable(int(on)))


def profile_read() -> dict:
    """{kernel name: (total ms, launches)} recorded since profile_enable(True)."""
    lib = load()
    out = {}
    for i in range(lib.elsaa_profile_count()):
        buf = C.create_string_buffer(128)
        ms, n = C.c_double(), C.c_int64()
        _check(lib.elsaa_profile_get(i, buf, 128, C.byref(ms), C.byref(n)))
        out[buf.value.decode()] = (ms.value, n.value)
    return out


def num_levels(cfg: Config) -> int:
    c = cfg.c()
    rc = load().elsaa_num_levels(C.byref(c))
    if rc < 0:
        _check(rc)
    return rc


def saved_bytes(cfg: Config) -> int:
    c, n = cfg.c(), C.c_size_t()
    _check(load().elsaa_saved_bytes(C.byref(c), C.byref(n)))
    return n.value


def workspace_bytes(cfg: Config, backward: bool = False) -> int:
    c, n = cfg.c(), C.c_size_t()
    _check(load().elsaa_workspace_bytes(C.byref(c), int(backward), C.byref(n)))
    return n.value


def saved_layout(cfg: Config) -> dict:
    c, L = cfg.c(), _SavedLayout()
    _check(load().elsaa_get_saved_layout(C.byref(c), C.byref(L)))
    return {f: getattr(L, f) for f, _ in _SavedLayout._fields_}


def perm_length(cfg: Config) -> int:
    """Entries of perm_q / perm_k per (b, h) (see elsaa_perm_length)."""
    c = cfg.c()
    n = load().elsaa_perm_length(C.byref(c))
    if n < 0:
        _check(int(n))
    return n


def _perm_shape(cfg: Config):
    """[B, H, Lv, N/2] for causal lists without padding, [B, H, P] with it,
    [B, H, N] non-causal."""
    if cfg.causal:
        lv, p = num_levels(cfg), perm_length(cfg)
        if lv * (cfg.N // 2) == p and cfg.N % 2 == 0:
            return (cfg.B, cfg.H, lv, cfg.N // 2)
        return (cfg.B, cfg.H, p)
    return (cfg.B, cfg.H, cfg.N)


def saved_views(cfg: Config, saved: torch.Tensor) -> dict:
    """Typed views into ``saved``: perm_q, perm_k, m, o_sparse, o_lowrank."""
    L = saved_layout(cfg)
    B, H, N, d = cfg.B, cfg.H, cfg.N, cfg.d_h
    ps = _perm_shape(cfg)
    npm = 1
    for x in ps:
        npm *= x

    def view(off, count, dtype, shape):
        nbytes = count * (torch.finfo(dtype).bits // 8 if dtype.is_floating_point else torch.iinfo(dtype).bits // 8)
        return saved[off:off + nbytes].view(dtype).view(*shape)

    return {
        "perm_q": view(L["perm_q"], npm, torch.int32, ps),
        "perm_k": view(L["perm_k"], npm, torch.int32, ps),
        "m": view(L["m"], B * H * N, torch.float32, (B, H, N)),
        "o_sparse": view(L["o_sparse"], B * H * N * d, torch.float32, (B, H, N, d)),
        "o_lowrank": view(L["o_lowrank"], B * H * N * d, cfg.torch_dtype, (B, H, N, d)),
    }


def _check_tensor(name, t, shape, dtype, dev):
    if t.shape != torch.Size(shape) or t.dtype != dtype or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)} on {dev}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def _check_inputs(cfg, q, k, v, w_sort, w_race, gates=None, extra=(), lam_rows=None):
    dev = q.device
    shp = (cfg.B, cfg.H, cfg.N, cfg.d_h)
    for name, t in (("q", q), ("k", k), ("v", v)) + tuple(extra):
        _check_tensor(name, t, shp, cfg.torch_dtype, dev)
    if w_sort is not None:
        _check_tensor("w_sort", w_sort, (cfg.H, cfg.sort_bits, cfg.d_h), torch.float32, dev)
    if w_race is not None:
        _check_tensor("w_race", w_race, (cfg.H, cfg.r >> cfg.race_bits, cfg.race_bits, cfg.d_h),
                      torch.float32, dev)
    if gates is not None:
        _check_tensor("gates", gates, (cfg.B, cfg.H, cfg.N, 2), torch.float32, dev)
    if lam_rows is not None:
        _check_tensor("lam_rows", lam_rows, (cfg.B, cfg.H, cfg.N), torch.float32, dev)
    return dev


class Buffers:
    """Preallocated outputs, saved state and workspaces for repeated calls."""

    def __init__(self, cfg: Config, device, backward: bool = True):
        B, H, N, d = cfg.B, cfg.H, cfg.N, cfg.d_h
        dt = cfg.torch_dtype
        self.o = torch.empty(B, H, N, d, dtype=dt, device=device)
        self.lse = torch.empty(B, H, N, dtype=torch.float32, device=device)
        self.d_lr = torch.empty(B, H, N, dtype=torch.float32, device=device)
        self.saved = torch.empty(saved_bytes(cfg), dtype=torch.uint8, device=device)
        ws = workspace_bytes(cfg, False)
        if backward:
            ws = max(ws, workspace_bytes(cfg, True))
            self.dq = torch.empty(B, H, N, d, dtype=dt, device=device)
            self.dk = torch.empty(B, H, N, d, dtype=dt, device=device)
            self.dv = torch.empty(B, H, N, d, dtype=dt, device=device)
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=device)


def select(cfg: Config, q, k, w_sort, workspace: Optional[torch.Tensor] = None):
    """Sorted index lists (perm_q, perm_k) of the sortLSH selection."""
    dev = _check_inputs(cfg, q, k, k, w_sort, None)
    ps = _perm_shape(cfg)
    pq = torch.empty(ps, dtype=torch.int32, device=dev)
    pk = torch.empty(ps, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = torch.empty(max(workspace_bytes(cfg), 256), dtype=torch.uint8, device=dev)
    c = cfg.c()
    _check(load().elsaa_select(C.byref(c), _p(q), _p(k), _p(w_sort), _p(pq), _p(pk), _p(workspace),
                               workspace.numel(), _stream(dev)))
    return pq, pk


def select_noalloc(cfg: Config, q, k, w_sort, perm_q: torch.Tensor, perm_k: torch.Tensor):
    """The selection into the caller's perm_q, perm_k through
    elsaa_select_noalloc (no allocation: the library's fixed scratch)."""
    dev = _check_inputs(cfg, q, k, k, w_sort, None)
    ps = _perm_shape(cfg)
    _check_tensor("perm_q", perm_q, ps, torch.int32, dev)
    _check_tensor("perm_k", perm_k, ps, torch.int32, dev)
    c = cfg.c()
    _check(load().elsaa_select_noalloc(C.byref(c), _p(q), _p(k), _p(w_sort), _p(perm_q), _p(perm_k),
                                       _stream(dev)))
    return perm_q, perm_k


def fwd(cfg: Config, q, k, v, w_sort, w_race, gates=None, buffers: Optional[Buffers] = None,
        lam_rows=None):
    """Forward; returns (o, lse, d_lr, saved).  lam_rows: per-token lambda_i
    [B, H, N] float32 (None: the scalar cfg.lam)."""
    dev = _check_inputs(cfg, q, k, v, w_sort, w_race, gates, lam_rows=lam_rows)
    bufs = buffers or Buffers(cfg, dev, backward=False)
    c = cfg.c()
    _check(load().elsaa_fwd(C.byref(c), _p(q), _p(k), _p(v), _p(w_sort), _p(w_race), _p(gates),
                            _p(lam_rows), _p(bufs.o), _p(bufs.lse), _p(bufs.d_lr), _p(bufs.saved),
                            bufs.saved.numel(), _p(bufs.workspace), bufs.workspace.numel(),
                            _stream(dev)))
    return bufs.o, bufs.lse, bufs.d_lr, bufs.saved


def bwd(cfg: Config, q, k, v, w_race, do, lse, d_lr, saved, gates=None, want_dgates=False,
        buffers: Optional[Buffers] = None, lam_rows=None, want_dlambda=False):
    """Backward; returns (dq, dk, dv), followed by dgates [B, H, N, 2] when
    want_dgates and by dlambda [B, H, N] when want_dlambda."""
    dev = _check_inputs(cfg, q, k, v, None, w_race, gates, extra=(("do", do),), lam_rows=lam_rows)
    bufs = buffers
    if bufs is None:
        bufs = Buffers(cfg, dev, backward=True)
    dg = torch.empty(cfg.B, cfg.H, cfg.N, 2, dtype=torch.float32, device=dev) if want_dgates else None
    dl = torch.empty(cfg.B, cfg.H, cfg.N, dtype=torch.float32, device=dev) if want_dlambda else None
    c = cfg.c()
    _check(load().elsaa_bwd(C.byref(c), _p(q), _p(k), _p(v), None, _p(w_race), _p(gates),
                            _p(lam_rows), _p(do), _p(lse), _p(d_lr), _p(saved), saved.numel(),
                            _p(bufs.dq), _p(bufs.dk), _p(bufs.dv), _p(dg), _p(dl),
                            _p(bufs.workspace), bufs.workspace.numel(), _stream(dev)))
    return (bufs.dq, bufs.dk, bufs.dv) + ((dg,) if want_dgates else ()) + ((dl,) if want_dlambda else ())


# ---------------------------------------------------------------------------
# dense projections (elsaa_gemm)
# ---------------------------------------------------------------------------
def _matrix(name, t):
    """(rows, cols, ld, heads, seq) of a stored operand: a 2-D tensor with unit
    column stride (plain) or a contiguous 4-D [B, H, S, dh] tensor (head-major,
    logical rows B*S and columns H*dh)."""
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    if t.dim() == 2:
        if t.stride(1) != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")
        return t.shape[0], t.shape[1], t.stride(0), 0, 0
    if t.dim() == 4:
        if not t.is_contiguous():
            raise ValueError(f"{name}: head-major operands must be contiguous [B, H, S, dh]")
        Bb, H, S, dh = t.shape
        return Bb * S, H * dh, 0, H, S
    raise ValueError(f"{name}: expected a 2-D matrix or a 4-D [B, H, S, dh] tensor")


def gemm_plan(a, b, trans_a=False, trans_b=False, out=None):
    """Descriptor of out = op(a) op(b) (see gemm)."""
    ar, ac, lda, ah, aseq = _matrix("a", a)
    br, bc, ldb, bh, bseq = _matrix("b", b)
    M, K = (ac, ar) if trans_a else (ar, ac)
    K2, N = (bc, br) if trans_b else (br, bc)
    if K != K2:
        raise ValueError(f"inner dimensions differ: {K} vs {K2}")
    cr, cc, ldc, ch, cseq = _matrix("out", out) if out is not None else (M, N, N, 0, 0)
    if (cr, cc) != (M, N):
        raise ValueError(f"out: expected a {M} x {N} matrix, got {cr} x {cc}")
    seqs = {s for s in (aseq, bseq, cseq) if s}
    if len(seqs) > 1:
        raise ValueError(f"head-major operands with different sequence lengths {sorted(seqs)}")
    seq = seqs.pop() if seqs else 0
    c_dtype = BF16 if out is None or out.dtype == torch.bfloat16 else F32
    return _GemmDesc(M, N, K, int(trans_a), int(trans_b), lda, ldb, ldc, ah, bh, ch, seq, c_dtype)


def gemm_workspace_bytes(desc: _GemmDesc) -> int:
    n = C.c_size_t()
    _check(load().elsaa_gemm_workspace_bytes(C.byref(desc), C.byref(n)))
    return n.value


def gemm(a, b, trans_a=False, trans_b=False, out=None, out_dtype=torch.bfloat16,
         workspace: Optional[torch.Tensor] = None):
    """out = op(a) @ op(b) on the matrix cores: bfloat16 operands, float32
    accumulation, op(x) = x.T when trans_x.  Operands and `out` are 2-D
    matrices (unit column stride) or contiguous head-major [B, H, S, dh]
    tensors standing for the [B*S, H*dh] matrix.  Without `out`, a plain
    [M, N] tensor of out_dtype is allocated."""
    if a.dtype != torch.bfloat16 or b.dtype != torch.bfloat16:
        raise ValueError("gemm operands must be bfloat16")
    if a.device != b.device:
        raise ValueError("operands on different devices")
    desc = gemm_plan(a, b, trans_a, trans_b, out)
    if out is None:
        out = torch.empty(desc.M, desc.N, dtype=out_dtype, device=a.device)
        desc.ldc = desc.N
        desc.c_dtype = BF16 if out_dtype == torch.bfloat16 else F32
    ws = gemm_workspace_bytes(desc)
    if ws and (workspace is None or workspace.numel() < ws):
        workspace = torch.empty(ws, dtype=torch.uint8, device=a.device)
    _check(load().elsaa_gemm(C.byref(desc), _p(a), _p(b), _p(out), _p(workspace) if ws else None,
                             workspace.numel() if ws else 0, _stream(a.device)))
    return out


# ---------------------------------------------------------------------------
# token-wise rules: gate network and query-dependent lambda
# ---------------------------------------------------------------------------
@dataclasses.dataclass
class TokenRules:
    """Parameters of the gate network (W1 [H, G, d_h], b1 [H, G], W2 [H, 2, G],
    b2 [H, 2]) and of the lambda rule (lam_w [H, d_h], lam_b [H], lam_c [H]),
    float32 tensors on the device; leave a rule's tensors None to switch it off."""
    W1: Optional[torch.Tensor] = None
    b1: Optional[torch.Tensor] = None
    W2: Optional[torch.Tensor] = None
    b2: Optional[torch.Tensor] = None
    lam_w: Optional[torch.Tensor] = None
    lam_b: Optional[torch.Tensor] = None
    lam_c: Optional[torch.Tensor] = None
    lambda_min: float = 1e-6

    @property
    def gate_hidden(self) -> int:
        return 0 if self.W1 is None else self.W1.shape[1]

    @property
    def has_lambda(self) -> bool:
        return self.lam_w is not None

    def c(self, cfg: Config) -> _TokenRules:
        H, d = cfg.H, cfg.d_h
        G = self.gate_hidden
        dev = None
        if G:
            for name, t, shp in (("W1", self.W1, (H, G, d)), ("b1", self.b1, (H, G)),
                                 ("W2", self.W2, (H, 2, G)), ("b2", self.b2, (H, 2))):
                _check_tensor(name, t, shp, torch.float32, t.device if dev is None else dev)
                dev = t.device
        if self.has_lambda:
            for name, t, shp in (("lam_w", self.lam_w, (H, d)), ("lam_b", self.lam_b, (H,)),
                                 ("lam_c", self.lam_c, (H,))):
                _check_tensor(name, t, shp, torch.float32, t.device if dev is None else dev)
                dev = t.device
        return _TokenRules(G, _p(self.W1), _p(self.b1), _p(self.W2), _p(self.b2), int(self.has_lambda),
                           _p(self.lam_w), _p(self.lam_b), _p(self.lam_c), self.lambda_min)


def token_rules_fwd(cfg: Config, rules: TokenRules, q):
    """(gates [B, H, N, 2] or None, lambda_rows [B, H, N] or None) of the rules."""
    dev = _check_inputs(cfg, q, q, q, None, None)
    gates = torch.empty(cfg.B, cfg.H, cfg.N, 2, dtype=torch.float32, device=dev) if rules.gate_hidden else None
    lam = torch.empty(cfg.B, cfg.H, cfg.N, dtype=torch.float32, device=dev) if rules.has_lambda else None
    c, r = cfg.c(), rules.c(cfg)
    _check(load().elsaa_token_rules_fwd(C.byref(c), C.byref(r), _p(q), _p(gates), _p(lam), _stream(dev)))
    return gates, lam


def token_rules_workspace_bytes(cfg: Config, rules: TokenRules) -> int:
    """Bytes of the backward's partial-sum workspace (one record per workgroup)."""
    c, r = cfg.c(), rules.c(cfg)
    n = C.c_size_t()
    _check(load().elsaa_token_rules_workspace_bytes(C.byref(c), C.byref(r), C.byref(n)))
    return n.value


def token_rules_bwd(cfg: Config, rules: TokenRules, q, dgates=None, dlambda=None, dq=None,
                    workspace: Optional[torch.Tensor] = None):
    """Parameter gradients of the rules (dict of tensors shaped like the
    parameters); when dq is given, the gate network's gradient with respect
    to q is added to it in place."""
    dev = _check_inputs(cfg, q, q, q, None, None)
    G = rules.gate_hidden
    if G:
        _check_tensor("dgates", dgates, (cfg.B, cfg.H, cfg.N, 2), torch.float32, dev)
    if rules.has_lambda:
        _check_tensor("dlambda", dlambda, (cfg.B, cfg.H, cfg.N), torch.float32, dev)
    if dq is not None:
        _check_tensor("dq", dq, (cfg.B, cfg.H, cfg.N, cfg.d_h), cfg.torch_dtype, dev)
    H, d = cfg.H, cfg.d_h
    f = lambda *shp: torch.empty(*shp, dtype=torch.float32, device=dev)   # noqa: E731
    out = {}
    if G:
        out.update(dW1=f(H, G, d), db1=f(H, G), dW2=f(H, 2, G), db2=f(H, 2))
    if rules.has_lambda:
        out.update(dlam_w=f(H, d), dlam_b=f(H), dlam_c=f(H))
    c, r = cfg.c(), rules.c(cfg)
    lib = load()
    need = token_rules_workspace_bytes(cfg, rules)
    ws = workspace if workspace is not None and workspace.numel() >= need else \
        torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    g = out.get
    _check(lib.elsaa_token_rules_bwd(C.byref(c), C.byref(r), _p(q), _p(dgates if G else None),
                                     _p(dlambda if rules.has_lambda else None), _p(dq),
                                     _p(g("dW1")), _p(g("db1")), _p(g("dW2")), _p(g("db2")),
                                     _p(g("dlam_w")), _p(g("dlam_b")), _p(g("dlam_c")),
                                     _p(ws), ws.numel(), _stream(dev)))
    return out


# ---------------------------------------------------------------------------
# around the operator: norm of the residual stream, 8-bit rows and products
# ---------------------------------------------------------------------------
def _gpu(name, t, dev=None, dtype=None):
    """Check that t is a tensor on a GPU (on `dev`, of `dtype`)."""
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a tensor on the GPU, got one on {t.device}")
    if dev is not None and t.device != dev:
        raise ValueError(f"{name}: expected a tensor on {dev}, got one on {t.device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")


def _vector(name, t, n, dev):
    """Check a contiguous float32 vector of n values on dev."""
    if t.dtype == torch.float32 and t.shape == (n,) and t.device == dev and t.is_contiguous():
        return
    _gpu(name, t, dev, torch.float32)
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous vector of {n} values, got {tuple(t.shape)}")


def _storage(name, t):
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise ValueError(f"{name}: unsupported dtype {t.dtype}")


def _rows(name, t, dev=None, dtype=None, shape=None):
    """(rows, cols, row stride) of a 2-D tensor with unit column stride, or of a
    contiguous tensor of any leading dimensions."""
    shp = t.shape
    if (len(shp) == 2 and t.is_cuda and (dev is None or t.device == dev) and (dtype is None or t.dtype == dtype)
            and (shape is None or shp == shape)):
        rows, cols = shp
        ld, unit = t.stride()
        if unit == 1 and ld >= cols:
            return rows, cols, ld
    _gpu(name, t, dev, dtype)
    if shape is not None and shp != shape:
        raise ValueError(f"{name}: expected {tuple(shape)}, got {tuple(shp)}")
    if len(shp) == 2:
        rows, cols = shp
        ld, unit = t.stride()
        if unit == 1 or cols == 1:
            return rows, cols, ld if rows > 1 or ld > cols else cols
    if len(shp) >= 1 and t.is_contiguous():
        cols = shp[-1]
        return (t.numel() // cols if cols else 0), cols, cols
    raise ValueError(f"{name}: expected a 2-D tensor with unit column stride or a contiguous tensor, "
                     f"got strides {tuple(t.stride())}")


def _workspace(ws, need, dev):
    """The caller's workspace if it is large enough, else a new one."""
    if ws is not None:
        _gpu("workspace", ws, dev, torch.uint8)
        if ws.numel() >= need and ws.is_contiguous():
            return ws
    return torch.empty(max(need, 256), dtype=torch.uint8, device=dev)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _launch(dev, fn, *args):
    """fn(*args, stream) on torch's current stream of dev, with dev current.
    (A call on a few tokens is shorter than a device guard and a stream
    object take, so both are made only where they are needed.)"""
    if dev.index == torch.cuda.current_device():
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev.index))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev.index))
    if rc != 0:
        _check(rc)


def _empty_rows8(rows, cols, dev):
    """A rows x cols 8-bit matrix whose row stride is a multiple of 16 (what gemm_i8 reads)."""
    return torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device=dev)[:, :cols]


def _rms_norm(x, weight, residual, eps, y, scale, sum_):
    dev, shp = x.device, x.shape
    rows, cols, ldx = _rows("x", x)
    dt = _storage("x", x)
    _vector("weight", weight, cols, dev)
    ldr = _rows("residual", residual, dev, x.dtype, shp)[2] if residual is not None else 0
    lds = _rows("out_sum", sum_, dev, x.dtype, shp)[2] if sum_ is not None else 0
    if scale is None:
        ydt, ldy = dt, _rows("out", y, dev, x.dtype, shp)[2]
    else:
        ydt, ldy = I8, _rows("out", y, dev, torch.int8, (rows, cols))[2]
        _vector("out_scale", scale, rows, dev)
    d = _NormDesc(rows, cols, dt, ydt, eps, ldx, ldr, lds, ldy)
    _launch(dev, load().elsaa_rms_norm_fwd, C.byref(d), _ptr(x), _ptr(residual), _ptr(weight), _ptr(sum_), _ptr(y),
            _ptr(scale))


def rms_norm_fwd(x, weight, residual=None, eps=1e-6, out=None, out_sum=None):
    """(y, s): s = x + residual, y = s / sqrt(mean(s^2) + eps) * weight over the
    last dimension.  x and residual bfloat16 or float32, weight float32; y and
    s in x's type, s None without a residual (unless out_sum is given).
    out_sum and out may each be x or residual, but not the same one."""
    _gpu("x", x)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if out_sum is None and residual is not None:
        out_sum = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _rms_norm(x, weight, residual, eps, out, None, out_sum)
    return out, out_sum


def rms_norm_i8(x, weight, residual=None, eps=1e-6, out=None, out_scale=None, out_sum=None):
    """(q, scale, s): the norm of rms_norm_fwd as 8-bit rows, y ~ q * scale[:, None]
    (scale = largest |y| of the row / 127), ready for gemm_i8.  q is a
    [rows, cols] matrix whatever the leading dimensions of x."""
    _gpu("x", x)
    rows, cols, _ = _rows("x", x)
    if out is None:
        out = _empty_rows8(rows, cols, x.device)
    if out_scale is None:
        out_scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    if out_sum is None and residual is not None:
        out_sum = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _rms_norm(x, weight, residual, eps, out, out_scale, out_sum)
    return out, out_scale, out_sum


def rms_norm_workspace_bytes(rows: int, cols: int) -> int:
    """Bytes of rms_norm_bwd's workspace (partial sums of the weight gradient)."""
    d, n = _NormDesc(rows, cols, BF16, BF16, 1e-6, cols, cols, cols, cols), C.c_size_t()
    _check(load().elsaa_rms_norm_workspace_bytes(C.byref(d), C.byref(n)))
    return n.value


def rms_norm_bwd(s, weight, dy, dsum=None, eps=1e-6, out=None, out_dweight=None, want_dweight=True,
                 workspace: Optional[torch.Tensor] = None):
    """(dx, dweight) of rms_norm_fwd at the stored sum s (x itself without a
    residual): dx, the gradient of x and of the residual alike, includes the
    residual stream's own gradient dsum when given.  dweight is float32 (None
    unless want_dweight)."""
    dev = s.device
    rows, cols, ldx = _rows("s", s)
    dt = _storage("s", s)
    _vector("weight", weight, cols, dev)
    ldy = _rows("dy", dy, dev, s.dtype, s.shape)[2]
    ldr = _rows("dsum", dsum, dev, s.dtype, s.shape)[2] if dsum is not None else 0
    if out is None:
        out = torch.empty(s.shape, dtype=s.dtype, device=dev)
    lds = _rows("out", out, dev, s.dtype, s.shape)[2]
    d = _NormDesc(rows, cols, dt, dt, eps, ldx, ldr, lds, ldy)
    dw, ws = None, None
    if want_dweight:
        dw = torch.empty(cols, dtype=torch.float32, device=dev) if out_dweight is None else out_dweight
        _vector("out_dweight", dw, cols, dev)
        ws = _workspace(workspace, rms_norm_workspace_bytes(rows, cols), dev)
    _launch(dev, load().elsaa_rms_norm_bwd, C.byref(d), _ptr(s), _ptr(weight), _ptr(dy), _ptr(dsum), _ptr(out),
            _ptr(dw), _ptr(ws), ws.numel() if ws is not None else 0)
    return out, dw


def quantize_rows(x, out=None, out_scale=None):
    """(q, scale): 8-bit rows of x with one float32 scale each, x ~ q * scale[:, None].
    x is a 2-D matrix (unit column stride) or a contiguous head-major
    [B, H, S, dh] tensor standing for the [B*S, H*dh] matrix.  Quantise a
    [N, K] weight (a row for each output channel) once for gemm_i8."""
    _gpu("x", x)
    dt = _storage("x", x)
    rows, cols, ld, heads, seq = _matrix("x", x)
    if out is None:
        out = _empty_rows8(rows, cols, x.device)
    if out_scale is None:
        out_scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    ldq = _rows("out", out, x.device, torch.int8, (rows, cols))[2]
    _vector("out_scale", out_scale, rows, x.device)
    d = _QuantDesc(rows, cols, dt, max(ld, cols) if rows == 1 else ld, ldq, heads, seq)
    _launch(x.device, load().elsaa_quantize_rows, C.byref(d), _ptr(x), _ptr(out), _ptr(out_scale))
    return out, out_scale


def gemm_i8_workspace_bytes(M: int, N: int, K: int) -> int:
    """Bytes of gemm_i8's workspace for an [M, K] x [N, K] product."""
    k16 = -(-K // 16) * 16
    d, n = _GemmI8Desc(M, N, K, k16, k16, N, 0, 0, BF16), C.c_size_t()
    _check(load().elsaa_gemm_i8_workspace_bytes(C.byref(d), C.byref(n)))
    return n.value


def _padding_held(name, t, K, ld):
    """Check that the last row's bytes up to the next multiple of 16, which gemm_i8
    reads and ignores, lie in t's storage as every other row's do (other strides
    and addresses are refused by the library)."""
    if ld % 16 or t.data_ptr() % 16:
        return
    end = t.storage_offset() + (t.shape[0] - 1) * ld + -(-K // 16) * 16
    if t.shape[0] and end > t.untyped_storage().nbytes():
        raise ValueError(f"{name}: rows of {K} bytes are read up to a multiple of 16, and the last one ends with its storage")


def gemm_i8(a, a_scale, b, b_scale, out=None, out_dtype=torch.bfloat16, workspace: Optional[torch.Tensor] = None):
    """out_ij = a_scale_i b_scale_j sum_k a_ik b_jk: 8-bit rows a [M, K] (tokens)
    and b [N, K] (a row for each output channel) with float32 scales, exact
    32-bit sums.  Row strides are multiples of 16 and rows are read up to a
    multiple of 16 (quantize_rows and rms_norm_i8 allocate them so).  `out` is a 2-D matrix (unit column stride)
    or a contiguous head-major [B, H, S, dh] tensor; without it a plain [M, N] tensor of
    out_dtype is allocated."""
    dev = a.device
    if a.dim() != 2 or b.dim() != 2:
        raise ValueError("a and b must be 2-D")
    M, K, lda = _rows("a", a, None, torch.int8)
    N, K2, ldb = _rows("b", b, dev, torch.int8)
    if K != K2:
        raise ValueError(f"inner dimensions differ: {K} vs {K2}")
    if K % 16:
        _padding_held("a", a, K, lda)
        _padding_held("b", b, K, ldb)
    _vector("a_scale", a_scale, M, dev)
    _vector("b_scale", b_scale, N, dev)
    if out is None:
        out = torch.empty(M, N, dtype=out_dtype, device=dev)
    _gpu("out", out, dev)
    c_dtype = _storage("out", out)
    cr, cc, ldc, ch, cseq = _matrix("out", out)
    if (cr, cc) != (M, N):
        raise ValueError(f"out: expected a {M} x {N} matrix, got {cr} x {cc}")
    d = _GemmI8Desc(M, N, K, lda, ldb, max(ldc, N) if M == 1 else ldc, ch, cseq, c_dtype)
    n = C.c_size_t()
    _check(load().elsaa_gemm_i8_workspace_bytes(C.byref(d), C.byref(n)))
    ws = _workspace(workspace, n.value, dev) if n.value else None
    _launch(dev, load().elsaa_gemm_i8, C.byref(d), _ptr(a), _ptr(a_scale), _ptr(b), _ptr(b_scale), _ptr(out),
            _ptr(ws), ws.numel() if ws is not None else 0)
    return out


# ---------------------------------------------------------------------------
# linear attention with a decay for each head
# ---------------------------------------------------------------------------
@dataclasses.dataclass
class DecayConfig:
    """Settings of the decay attention (see elsaa_decay_desc in include/elsaa.h)."""
    B: int
    H: int
    N: int
    d_h: int
    dtype: str = "bf16"     # storage type of q, k, v, o and their gradients
    scale: float = 0.0      # <= 0 -> 1/sqrt(d_h)

    def c(self) -> _DecayDesc:
        return _DecayDesc(self.B, self.H, self.N, self.d_h, BF16 if self.dtype == "bf16" else F32, self.scale)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32


def _batch_stride(name, t, B, H, N, dh):
    """Elements from one sequence to the next of a [B, H, N, dh] tensor (0: only one).
    (Sequences that lie over each other, as in an expanded tensor, have a stride of 0 too,
    which the library would take for contiguous ones.)"""
    if t.shape != (B, H, N, dh):
        raise ValueError(f"{name}: expected {(B, H, N, dh)}, got {tuple(t.shape)}")
    sb, sh, sn, se = t.stride()
    if se != 1 or (N > 1 and sn != dh) or (H > 1 and sh != N * dh):
        raise ValueError(f"{name}: the heads, tokens and values of a sequence must be contiguous")
    if B == 1:
        return 0
    if sb < H * N * dh:
        raise ValueError(f"{name}: sequences {sb} elements apart overlap (expanded tensors must be made contiguous)")
    return sb


def _decay_desc(cfg: DecayConfig, dev, **tensors):
    """Descriptor with the batch strides of the named [B, H, N, d_h] tensors."""
    d = cfg.c()
    B = cfg.B
    for name, t in tensors.items():
        _gpu(name, t, dev, cfg.torch_dtype)
        batch = _batch_stride(name, t, B, cfg.H, cfg.N, cfg.d_h)
        field = {"do": "o"}.get(name, name) + "_batch"
        if name == "do" and B > 1 and d.o_batch not in (0, batch):
            raise ValueError("o and do with different batch strides")
        setattr(d, field, batch)
    return d


def _decay_common(cfg, dev, log_decay, lengths, **states):
    _vector("log_decay", log_decay, cfg.H, dev)
    for name, t in states.items():
        if t is not None:
            _check_tensor(name, t, (cfg.B, cfg.H, cfg.d_h, cfg.d_h), torch.float32, dev)
    if lengths is not None:
        _check_tensor("lengths", lengths, (cfg.B,), torch.int32, dev)


def _decay_workspace(d: _DecayDesc, backward: bool) -> int:
    n = C.c_size_t()
    _check(load().elsaa_decay_workspace_bytes(C.byref(d), int(backward), C.byref(n)))
    return n.value


def decay_workspace_bytes(cfg: DecayConfig, backward: bool = False) -> int:
    return _decay_workspace(cfg.c(), backward)


def decay_fwd(cfg: DecayConfig, q, k, v, log_decay, state=None, lengths=None, out=None, out_state=None,
              want_state=True, workspace: Optional[torch.Tensor] = None, zero_tail=False):
    """(o, state): S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale q_t^T S_t
    over N tokens from `state` (None: zero); the returned state [B, H, d_h, d_h]
    float32 is the one behind the last token (None unless want_state).
    q, k, v are [B, H, N, d_h], each sequence contiguous (head ranges of one
    projection buffer will do); lengths int32 [B] shortens sequences: rows of o behind them are not written,
    or set to zero with zero_tail."""
    dev = q.device
    if out is None:
        out = torch.empty(cfg.B, cfg.H, cfg.N, cfg.d_h, dtype=cfg.torch_dtype, device=dev)
    if out_state is None and want_state:
        out_state = torch.empty(cfg.B, cfg.H, cfg.d_h, cfg.d_h, dtype=torch.float32, device=dev)
    d = _decay_desc(cfg, dev, q=q, k=k, v=v, o=out)
    d.zero_tail = int(zero_tail)
    _decay_common(cfg, dev, log_decay, lengths, state=state, out_state=out_state)
    ws = _workspace(workspace, _decay_workspace(d, False), dev)
    _launch(dev, load().elsaa_decay_fwd, C.byref(d), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(state),
            _ptr(lengths), _ptr(out), _ptr(out_state), _ptr(ws), ws.numel())
    return out, out_state


def decay_bwd(cfg: DecayConfig, q, k, v, log_decay, do, state=None, dstate_out=None, lengths=None, out=None,
              want_dstate=False, workspace: Optional[torch.Tensor] = None):
    """(dq, dk, dv, dstate) of decay_fwd for the upstream gradients do of o and
    dstate_out of the returned state (None: zero); dstate is the gradient of
    `state` (None unless want_dstate).  `out` may give (dq, dk, dv)."""
    dev = q.device
    shp = (cfg.B, cfg.H, cfg.N, cfg.d_h)
    dq, dk, dv = out if out is not None else (torch.empty(shp, dtype=cfg.torch_dtype, device=dev) for _ in range(3))
    d = _decay_desc(cfg, dev, q=q, k=k, v=v, do=do, dq=dq, dk=dk, dv=dv)
    dstate = torch.empty(cfg.B, cfg.H, cfg.d_h, cfg.d_h, dtype=torch.float32, device=dev) if want_dstate else None
    _decay_common(cfg, dev, log_decay, lengths, state=state, dstate_out=dstate_out)
    ws = _workspace(workspace, _decay_workspace(d, True), dev)
    _launch(dev, load().elsaa_decay_bwd, C.byref(d), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(do),
            _ptr(state), _ptr(dstate_out), _ptr(lengths), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dstate), _ptr(ws),
            ws.numel())
    return dq, dk, dv, dstate


def decay_step(cfg: DecayConfig, q, k, v, log_decay, state, out=None, out_state=None):
    """(o, state) of one token for each sequence (cfg.N = 1; q, k, v [B, H, 1, d_h]):
    the recurrent form of decay_fwd.  `state` moves on in place unless out_state is given."""
    dev = q.device
    if out is None:
        out = torch.empty(cfg.B, cfg.H, cfg.N, cfg.d_h, dtype=cfg.torch_dtype, device=dev)
    if out_state is None:
        out_state = state
    d = _decay_desc(cfg, dev, q=q, k=k, v=v, o=out)
    _decay_common(cfg, dev, log_decay, None, state=state, out_state=out_state)
    _launch(dev, load().elsaa_decay_step, C.byref(d), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(state),
            _ptr(out), _ptr(out_state))
    return out, out_state
