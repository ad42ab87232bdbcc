"""ctypes binding of libstrp.so: same entry-point names, argument marshalling only.

Every computation happens in the HIP library.  PyTorch is used for device memory and the
stream handle.  If the library has not been built, loading fails with an error (there is no
fallback path).
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libstrp.so")

OK, EINVAL, ENOMEM, ENOTPD, ENONFINITE, EHIP, ESTATE = range(7)
BF16, F32 = 0, 1
WANDA, LEMMA, GAIN = 0, 1, 2
SIDE_FC1, SIDE_FC2 = 0, 1
PREC_FAST, PREC_SPLIT = 0, 1
PROD_GRAM, PROD_RHS2, PROD_RHS1, PROD_RESID, PROD_AUPD, PROD_ZUPD = range(6)
STAGE_SELECT, STAGE_REFIT2, STAGE_REFIT1, STAGE_AUPD, STAGE_ZUPD, STAGE_OBJ = 1, 2, 4, 8, 16, 32
STAGE_ALL = 63
ACT_NONE, ACT_RELU, ACT_GELU = range(3)
CACHE_BF16, CACHE_F32, CACHE_Q4 = range(3)
TOP_MAX = 16

EXPORTS = [
    "strp_create", "strp_destroy", "strp_last_error", "strp_set_precision", "strp_set_product_planes", "strp_set_workspace", "strp_workspace_captured",
    "strp_poll", "strp_workspace_bytes", "strp_module_cache_bytes", "strp_profile_enable", "strp_profile_read", "strp_profile_launches", "strp_gram", "strp_score_alloc", "strp_mask_topk", "strp_mask_topk_static", "strp_topk_workspace_bytes", "strp_weight_energy", "strp_alloc_inverse", "strp_alloc_softmax",
    "strp_refit", "strp_module_init", "strp_admm_step",
    "strp_linear", "strp_linear_workspace_bytes", "strp_layer_norm", "strp_attention", "strp_token_logprobs", "strp_token_logprobs_workspace_bytes",
    "strp_cache_append", "strp_cache_attention", "strp_cache_attention_workspace_bytes",
    "strp_verify_draft", "strp_verify_draft_workspace_bytes",
]


class StrpError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"strp status {status}: {msg}")
        self.status = status


class ModuleDesc(C.Structure):
    _fields_ = [("d", C.c_int32), ("f", C.c_int32), ("T", C.c_int64), ("ldx", C.c_int64), ("lda", C.c_int64),
                ("x_dtype", C.c_int32), ("w_dtype", C.c_int32), ("k_max", C.c_int32)]


class ScoreIn(C.Structure):
    _fields_ = [("A", C.c_void_p), ("a_dtype", C.c_int32), ("Z", C.c_void_p), ("Z0", C.c_void_p), ("ld", C.c_int64),
                ("T", C.c_int64), ("n_channels", C.c_int32), ("group", C.c_int32), ("mode", C.c_int32),
                ("n2", C.c_void_p), ("What", C.c_void_p), ("w_dtype", C.c_int32), ("w_rows", C.c_int32),
                ("ldw", C.c_int64)]


class ModuleState(C.Structure):
    _fields_ = [("X", C.c_void_p), ("W1hat", C.c_void_p), ("W2hat", C.c_void_p), ("Z", C.c_void_p), ("A", C.c_void_p),
                ("Z0", C.c_void_p), ("Y", C.c_void_p), ("W1", C.c_void_p), ("W2", C.c_void_p), ("H", C.c_void_p),
                ("cholH", C.c_void_p), ("n2", C.c_void_p), ("score", C.c_void_p), ("mask", C.c_void_p),
                ("idx", C.c_void_p), ("scalars", C.c_void_p), ("cache", C.c_void_p), ("s", C.c_int32), ("iter", C.c_int32),
                ("sums_cached", C.c_int32), ("precision", C.c_int32)]


class Params(C.Structure):
    _fields_ = [("alpha", C.c_double), ("beta", C.c_double), ("delta", C.c_double), ("mode", C.c_int32),
                ("reselect", C.c_int32), ("k", C.c_int32), ("stages", C.c_int32)]


class Report(C.Structure):
    _fields_ = [("terms", C.c_double * 5), ("J", C.c_double), ("J_ridge", C.c_double), ("lam1", C.c_double),
                ("lam2", C.c_double), ("tau", C.c_float), ("s", C.c_int32), ("status", C.c_int32)]


class WeightRef(C.Structure):
    _fields_ = [("W", C.c_void_p), ("dtype", C.c_int32), ("rows", C.c_int32), ("cols", C.c_int32), ("ld", C.c_int64)]


class LinearIn(C.Structure):
    _fields_ = [("W", C.c_void_p), ("X", C.c_void_p), ("bias", C.c_void_p), ("R", C.c_void_p), ("Y", C.c_void_p),
                ("w_dtype", C.c_int32), ("x_dtype", C.c_int32), ("y_dtype", C.c_int32), ("M", C.c_int32), ("K", C.c_int32),
                ("act", C.c_int32), ("T", C.c_int64), ("ldw", C.c_int64), ("ldx", C.c_int64), ("ldr", C.c_int64), ("ldy", C.c_int64)]


class AttentionIn(C.Structure):
    _fields_ = [("Q", C.c_void_p), ("K", C.c_void_p), ("V", C.c_void_p), ("C", C.c_void_p), ("seq_start", C.c_void_p),
                ("kv_of_head", C.c_void_p), ("dtype", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("d_head", C.c_int32),
                ("n_seq", C.c_int32), ("scale", C.c_float), ("T", C.c_int64), ("ldq", C.c_int64), ("ldk", C.c_int64),
                ("ldv", C.c_int64), ("ldc", C.c_int64)]


class Cache(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("K_scale", C.c_void_p), ("V_scale", C.c_void_p), ("table", C.c_void_p), ("past", C.c_void_p),
                ("seq_start", C.c_void_p), ("format", C.c_int32), ("kv_heads", C.c_int32), ("d_head", C.c_int32), ("page", C.c_int32),
                ("pages", C.c_int32), ("n_seq", C.c_int32), ("ld_table", C.c_int32)]


class CacheAppendIn(C.Structure):
    _fields_ = [("cache", Cache), ("K", C.c_void_p), ("V", C.c_void_p), ("Q", C.c_void_p), ("Qr", C.c_void_p), ("inv_freq", C.c_void_p),
                ("dtype", C.c_int32), ("heads", C.c_int32), ("rot", C.c_int32), ("pairs", C.c_int32), ("T", C.c_int64), ("ldk", C.c_int64),
                ("ldv", C.c_int64), ("ldq", C.c_int64), ("ldqr", C.c_int64)]


class CacheAttentionIn(C.Structure):
    _fields_ = [("cache", Cache), ("Q", C.c_void_p), ("C", C.c_void_p), ("kv_of_head", C.c_void_p), ("dtype", C.c_int32), ("heads", C.c_int32),
                ("scale", C.c_float), ("T", C.c_int64), ("ldq", C.c_int64), ("ldc", C.c_int64)]


class VerifyDraftIn(C.Structure):
    _fields_ = [("target", C.c_void_p), ("draft", C.c_void_p), ("draft_id", C.c_void_p), ("u", C.c_void_p), ("u_next", C.c_void_p),
                ("draft_start", C.c_void_p), ("accepted", C.c_void_p), ("next_id", C.c_void_p), ("dtype", C.c_int32), ("V", C.c_int32),
                ("n_seq", C.c_int32), ("temperature", C.c_double), ("T", C.c_int64), ("ldt", C.c_int64), ("ldd", C.c_int64)]


# Their bytes from the fields in order: a call's cost on the host is the marshalling, and packing in one go is the cheaper form of it.
_LINEAR, _ATTENTION = struct.Struct("@5P6i5q"), struct.Struct("@6P5if5q")
assert _LINEAR.size == C.sizeof(LinearIn) and _ATTENTION.size == C.sizeof(AttentionIn)
_CACHE_APPEND, _CACHE_ATTENTION = struct.Struct("@7P7i4x5P4i5q"), struct.Struct("@7P7i4x3P2if4x3q")
_VERIFY_DRAFT = struct.Struct("@8P3i4xd3q")
assert _VERIFY_DRAFT.size == C.sizeof(VerifyDraftIn)
assert _CACHE_APPEND.size == C.sizeof(CacheAppendIn) and _CACHE_ATTENTION.size == C.sizeof(CacheAttentionIn)

_packers = {}


def _pack_refs(n):
    """bytes of an array of n WeightRef from its fields in order."""
    f = _packers.get(n)
    if f is None:
        packer = struct.Struct("@" + "Piii4xq" * n)
        assert packer.size == n * C.sizeof(WeightRef)
        f = _packers[n] = packer.pack
    return f


class ProfileEntry(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("launches", C.c_int32), ("ms", C.c_double), ("flops", C.c_double),
                ("bytes", C.c_double)]


_lib = None


def load_library():
    """dlopen libstrp.so (built in-tree by paper_2510_03246_amd/build.py); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} not built: run `python -m paper_2510_03246_amd.build` "
                                "(or __graft_entry__.build()); there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, dbl = C.c_void_p, C.c_int32, C.c_int64, C.c_double
    lib.strp_create.argtypes = [C.POINTER(vp), C.c_int, vp]
    lib.strp_destroy.argtypes = [vp]
    lib.strp_last_error.argtypes = [vp]
    lib.strp_last_error.restype = C.c_char_p
    lib.strp_set_precision.argtypes = [vp, C.c_int]
    lib.strp_set_product_planes.argtypes = [vp, C.c_int, i32, i32]
    lib.strp_set_workspace.argtypes = [vp, vp, C.c_size_t]
    lib.strp_workspace_captured.argtypes = [vp, i32]
    lib.strp_poll.argtypes = [vp]
    lib.strp_profile_enable.argtypes = [vp, C.c_int]
    lib.strp_profile_read.argtypes = [vp, C.POINTER(ProfileEntry), i32, C.POINTER(i32)]
    lib.strp_profile_launches.argtypes = [vp, C.POINTER(ProfileEntry), i32, C.POINTER(i32)]
    lib.strp_workspace_bytes.argtypes = [C.POINTER(ModuleDesc)]
    lib.strp_workspace_bytes.restype = C.c_size_t
    lib.strp_module_cache_bytes.argtypes = [C.POINTER(ModuleDesc)]
    lib.strp_module_cache_bytes.restype = C.c_size_t
    lib.strp_topk_workspace_bytes.restype = C.c_size_t
    lib.strp_topk_workspace_bytes.argtypes = [C.c_int32]
    lib.strp_weight_energy.argtypes = [vp, vp, i32, C.c_double, C.c_double, C.c_double, vp]
    lib.strp_alloc_inverse.argtypes = [vp, vp, i32, vp, vp, C.c_double, C.c_double, C.c_double, vp, vp]
    lib.strp_alloc_softmax.argtypes = [vp, vp, i32, vp, vp, C.c_double, C.c_double, C.c_double, vp, vp]
    lib.strp_gram.argtypes = [vp, vp, C.c_int, i32, i64, i64, vp, i32, vp, i32, vp, C.c_int]
    lib.strp_score_alloc.argtypes = [vp, C.POINTER(ScoreIn), vp, vp, i32, i32, vp, vp, dbl, dbl, dbl, vp, vp]
    lib.strp_mask_topk.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp]
    lib.strp_mask_topk_static.argtypes = [vp, vp, i32, i32, vp, vp, vp]
    lib.strp_refit.argtypes = [vp, C.c_int, vp, i32, dbl, vp, C.c_int, vp, C.c_int, i64, vp, C.c_int, i64, i64, vp,
                               i32, vp, i32, i32]
    lib.strp_module_init.argtypes = [vp, C.POINTER(ModuleDesc), C.POINTER(ModuleState), C.POINTER(Params)]
    lib.strp_admm_step.argtypes = [vp, C.POINTER(ModuleDesc), C.POINTER(ModuleState), C.POINTER(Params),
                                   C.POINTER(Report)]
    lib.strp_linear.argtypes = [vp, vp]               # LinearIn, or its bytes
    lib.strp_layer_norm.argtypes = [vp, vp, C.c_int, i32, i64, i64, vp, vp, dbl, vp, i64]
    lib.strp_attention.argtypes = [vp, vp]
    lib.strp_token_logprobs.argtypes = [vp, vp, C.c_int, i32, i64, i64, vp, vp, vp, i32, vp, vp, i64]
    lib.strp_cache_append.argtypes = [vp, vp]
    lib.strp_cache_attention.argtypes = [vp, vp]
    lib.strp_cache_attention_workspace_bytes.argtypes = [i32]
    lib.strp_cache_attention_workspace_bytes.restype = C.c_size_t
    lib.strp_verify_draft.argtypes = [vp, vp]
    lib.strp_verify_draft_workspace_bytes.argtypes = [i32, i64, i32]
    lib.strp_verify_draft_workspace_bytes.restype = C.c_size_t
    lib.strp_linear_workspace_bytes.argtypes = [i32, i32, i64, C.c_int, C.c_int]
    lib.strp_linear_workspace_bytes.restype = C.c_size_t
    lib.strp_token_logprobs_workspace_bytes.argtypes = [i32, i64, i32]
    lib.strp_token_logprobs_workspace_bytes.restype = C.c_size_t
    for name in EXPORTS:
        if not name.endswith("_bytes") and name != "strp_last_error":
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _ptr(t):
    return None if t is None else t.data_ptr()       # every pointer argument is declared c_void_p


_CODES = {torch.bfloat16: BF16, torch.float32: F32}


def dtype_code(t: torch.Tensor) -> int:
    try:
        return _CODES[t.dtype]
    except KeyError:
        raise TypeError(f"unsupported dtype {t.dtype}") from None


def aligned_rows(W: torch.Tensor) -> torch.Tensor:
    """W [M x K] as strp_linear reads weights, rows beginning at multiples of eight entries: W itself where they do, else the first K columns of
    a copy that is wider.  Done once, for weights as a refit leaves them or with columns taken out."""
    M, K = W.shape
    if W.stride(1) == 1 and W.stride(0) % 8 == 0 and W.stride(0) >= K and W.data_ptr() % 16 == 0:
        return W
    wide = torch.zeros((M, (K + 7) // 8 * 8), dtype=W.dtype, device=W.device)
    wide[:, :K] = W
    return wide[:, :K]


class Context:
    """Owns a strp_ctx bound to torch's current stream on `device`, plus the caller-side workspace.  Its calls are enqueued on that stream also where another
    one is current: then the caller orders the two, and keeps what the calls read until they have."""

    def __init__(self, device=0, workspace_bytes: int | None = None):
        self.lib = load_library()
        self.device = torch.device("cuda", device)
        self.index = self.device.index            # for the comparison in every call, where an attribute of an attribute costs twice
        torch.cuda.set_device(self.device)
        self.stream = torch.cuda.current_stream(self.device)
        h = C.c_void_p()
        st = self.lib.strp_create(C.byref(h), device, C.c_void_p(self.stream.cuda_stream))
        if st != OK:
            raise StrpError(st, "strp_create failed")
        self.h = h
        self.ws = None
        self.kept = []                            # workspaces that graphs have and that were replaced (forget_graphs)
        if workspace_bytes:
            self.set_workspace(workspace_bytes)

    def close(self):
        if self.h:
            self.lib.strp_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def check(self, st):
        if st != OK:
            raise StrpError(st, self.lib.strp_last_error(self.h).decode())

    # ---- plumbing ---------------------------------------------------------------------
    def set_workspace(self, nbytes: int):
        """A workspace of nbytes in place of the present one; a failure that has not been polled stays pending.  Not while the
        context's stream is being captured."""
        captured = self.lib.strp_workspace_captured(self.h, 0)
        with torch.cuda.stream(self.stream):
            ws = torch.empty(int(nbytes), dtype=torch.uint8, device=self.device)
            self.check(self.lib.strp_set_workspace(self.h, _ptr(ws), int(nbytes)))
            if self.ws is not None:
                ws[:4].copy_(self.ws[:4])         # the status word
        if captured:
            self.kept.append(self.ws)             # a graph that is replayed still writes there
        self.ws = ws

    def ensure_workspace(self, nbytes: int):
        if self.ws is None or self.ws.numel() < nbytes:
            self.set_workspace(nbytes)

    def forget_graphs(self):
        """No graph that has captured this context's calls is replayed any more: what was kept for them is freed, which otherwise lasts as
        long as the context (a context must outlive its graphs)."""
        self.lib.strp_workspace_captured(self.h, 1)
        self.kept.clear()

    def set_precision(self, prec: int):
        self.check(self.lib.strp_set_precision(self.h, prec))

    def set_product_planes(self, product: int, planes_p: int, planes_q: int):
        self.check(self.lib.strp_set_product_planes(self.h, product, planes_p, planes_q))

    def poll(self) -> int:
        return self.lib.strp_poll(self.h)

    def profile_enable(self, on: bool):
        self.check(self.lib.strp_profile_enable(self.h, int(on)))

    def profile_read(self):
        """Per-kernel-class totals since profile_enable: {name: dict(launches, ms, flops, bytes)}."""
        buf = (ProfileEntry * 64)()
        n = C.c_int32(0)
        self.check(self.lib.strp_profile_read(self.h, buf, 64, C.byref(n)))
        return {buf[i].name.decode(): dict(launches=buf[i].launches, ms=buf[i].ms, flops=buf[i].flops,
                                           bytes=buf[i].bytes) for i in range(n.value)}

    def profile_launches(self, max_entries: int = 4096):
        """The records since profile_enable one by one, in enqueue order: [(name, ms, flops, bytes), ...]."""
        buf = (ProfileEntry * max_entries)()
        n = C.c_int32(0)
        self.check(self.lib.strp_profile_launches(self.h, buf, max_entries, C.byref(n)))
        return [(buf[i].name.decode(), buf[i].ms, buf[i].flops, buf[i].bytes) for i in range(n.value)]

    def workspace_bytes(self, desc: ModuleDesc) -> int:
        return int(self.lib.strp_workspace_bytes(C.byref(desc)))

    # ---- entry points -------------------------------------------------------------------
    def strp_gram(self, A, T, idx=None, G=None, diag=None, accumulate=False, s=None):
        Crows, ldA = A.shape[0], A.stride(0)
        s = (idx.numel() if idx is not None else Crows) if s is None else s
        if G is None:
            G = torch.empty((s, s), dtype=torch.float32, device=A.device)
        self.check(self.lib.strp_gram(self.h, _ptr(A), dtype_code(A), Crows, T, ldA, _ptr(idx), s, _ptr(G),
                                      G.stride(0), _ptr(diag), int(accumulate)))
        return G

    def strp_score_alloc(self, A, T, mode, unit_score, energies, layer_idx, L, group=1, Z=None, Z0=None, n2=None,
                         What=None, n_units=None, group_id=None, rbar=0.5, temperature=1.0, rmax=0.95, r_out=None,
                         nprune_out=None):
        si = ScoreIn()
        si.A, si.a_dtype = A.data_ptr(), dtype_code(A)
        si.Z = Z.data_ptr() if Z is not None else None
        si.Z0 = Z0.data_ptr() if Z0 is not None else None
        si.ld, si.T, si.n_channels, si.group, si.mode = A.stride(0), T, A.shape[0], group, mode
        si.n2 = n2.data_ptr() if n2 is not None else None
        if What is not None:
            si.What, si.w_dtype, si.w_rows, si.ldw = What.data_ptr(), dtype_code(What), What.shape[0], What.stride(0)
        self.check(self.lib.strp_score_alloc(self.h, C.byref(si), _ptr(unit_score), _ptr(energies), layer_idx, L,
                                             _ptr(n_units), _ptr(group_id), rbar, temperature, rmax, _ptr(r_out),
                                             _ptr(nprune_out)))

    def strp_mask_topk(self, score, k, group=1, n=None):
        n = score.numel() if n is None else n
        mask = torch.empty(n, dtype=torch.uint8, device=score.device)
        idx = torch.empty(max(k * group, 1), dtype=torch.int32, device=score.device)
        tau = torch.empty(1, dtype=torch.float32, device=score.device)
        need = int(self.lib.strp_topk_workspace_bytes(n))
        if need:
            self.ensure_workspace(need)
        self.check(self.lib.strp_mask_topk(self.h, _ptr(score), n, k, group, _ptr(mask), _ptr(idx), _ptr(tau)))
        return mask, idx[: k * group], tau

    def strp_mask_topk_static(self, score, k, mask, idx, tau, n=None):
        """The allocation-free variant: every buffer, outputs included, is the caller's; nothing is allocated here."""
        n = score.numel() if n is None else n
        self.check(self.lib.strp_mask_topk_static(self.h, _ptr(score), n, k, _ptr(mask), _ptr(idx), _ptr(tau)))

    def strp_weight_energy(self, mats, var_coef, l2_coef, scale, energy):
        """energy (device double, 1 element) += scale (|W|_1 + var_coef Var(W) + l2_coef |W|_2) over the 2-D tensors in mats."""
        self.ensure_workspace(1 << 16)
        # a model has hundreds of small groups, so a call's cost is this marshalling: the WeightRef array is packed in one go
        args = []
        for m in mats:
            args += (m.data_ptr(), dtype_code(m), m.shape[0], m.shape[1], m.stride(0))
        refs = _pack_refs(len(mats))(*args)
        # float(): coefficients may be numpy scalars or one-element tensors, which ctypes does not take
        self.check(self.lib.strp_weight_energy(self.h, refs, len(mats), float(var_coef), float(l2_coef), float(scale), _ptr(energy)))

    def strp_alloc_inverse(self, energies, n_units, rbar, temperature, rmax=0.95, group_id=None):
        L = energies.numel()
        r = torch.empty(L, dtype=torch.float64, device=energies.device)
        npr = torch.empty(L, dtype=torch.int32, device=energies.device)
        self.check(self.lib.strp_alloc_inverse(self.h, _ptr(energies), L, _ptr(n_units), _ptr(group_id), float(rbar),
                                               float(temperature), float(rmax), _ptr(r), _ptr(npr)))
        return r, npr

    def strp_alloc_softmax(self, energies, n_units, rbar, temperature, rmax=0.95, group_id=None):
        L = energies.numel()
        r = torch.empty(L, dtype=torch.float64, device=energies.device)
        npr = torch.empty(L, dtype=torch.int32, device=energies.device)
        self.check(self.lib.strp_alloc_softmax(self.h, _ptr(energies), L, _ptr(n_units), _ptr(group_id), float(rbar),
                                               float(temperature), float(rmax), _ptr(r), _ptr(npr)))
        return r, npr

    def strp_refit(self, side, Gram, lam, Lhs, Rhs, T, idx, W, chol=None, chol_valid=False):
        out, inn = W.shape
        self.check(self.lib.strp_refit(self.h, side, _ptr(Gram), Gram.stride(0) if Gram is not None else 0, float(lam),
                                       _ptr(chol), int(chol_valid), _ptr(Lhs), dtype_code(Lhs), Lhs.stride(0),
                                       _ptr(Rhs), dtype_code(Rhs), Rhs.stride(0), T, _ptr(idx), idx.numel(), _ptr(W),
                                       out, inn))
        return W

    # ---- a decoder layer's forward operators ----------------------------------------------
    # Activations are [channels x ld] tensors with the tokens contiguous, T of the ld columns valid; what the library cannot see
    # (shapes, strides, types and devices of the tensors) is checked here, the rest there.
    def _matrix(self, name, t, rows, cols, dtypes):
        """Leading dimension of t as an operand of `rows` rows and at least `cols` columns, of one of the dtypes, on this context's device."""
        shape = t.shape
        if t.get_device() != self.index:
            raise ValueError(f"{name} is on {t.device}, the context on {self.device}")
        if t.dtype not in dtypes:
            raise TypeError(f"{name}: unsupported dtype {t.dtype}")
        if len(shape) != 2 or shape[0] != rows or shape[1] < cols:
            raise ValueError(f"{name}: shape {tuple(shape)}, needs ({rows}, at least {cols})")
        ld, step = t.stride()
        if step != 1 and shape[1] > 1:
            raise ValueError(f"{name}: its rows are not contiguous")
        # torch may report anything as the stride of a single row
        return shape[1] if rows == 1 and (ld < shape[1] or ld % 8) else ld

    def _vector(self, name, t, n, dtype):
        """Address of a contiguous vector of at least n entries; 0 for None."""
        if t is None:
            return 0
        if t.get_device() != self.index:
            raise ValueError(f"{name} is on {t.device}, the context on {self.device}")
        if t.dtype is not dtype:
            raise TypeError(f"{name}: {t.dtype}, needs {dtype}")
        shape = t.shape
        if len(shape) != 1 or shape[0] < n or (n > 1 and not t.is_contiguous()):
            raise ValueError(f"{name}: needs {n} contiguous entries")
        return t.data_ptr()

    def _empty(self, shape, dtype):
        """An output, from the memory of the stream that writes it."""
        if torch.cuda.current_stream(self.device) == self.stream:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _new(self, rows, T, dtype):
        return self._empty((rows, (T + 7) // 8 * 8), dtype)

    def strp_linear(self, W, X, T, bias=None, act=ACT_NONE, residual=None, out=None):
        """act(W X + bias) + residual: W [M x K] with rows at multiples of eight entries (aligned_rows), X [K x ld], bias [M] fp32, residual
        [M x ld] of out's dtype (out itself is allowed).  Returns out, made in X's dtype where none is given."""
        M, K = W.shape
        if out is None:
            out = self._new(M, T, X.dtype)
        ldw, ldx, ldy = self._matrix("W", W, M, K, _CODES), self._matrix("X", X, K, T, _CODES), self._matrix("out", out, M, T, _CODES)
        w, x, y = _CODES[W.dtype], _CODES[X.dtype], _CODES[out.dtype]
        r, ldr = (0, 0) if residual is None else (residual.data_ptr(), self._matrix("residual", residual, M, T, (out.dtype,)))
        need = self.lib.strp_linear_workspace_bytes(M, K, T, w, x)
        if need:
            self.ensure_workspace(need)
        self.check(self.lib.strp_linear(self.h, _LINEAR.pack(W.data_ptr(), X.data_ptr(), self._vector("bias", bias, M, torch.float32), r, out.data_ptr(),
                                                             w, x, y, M, K, act, T, ldw, ldx, ldr, ldy)))
        return out

    def strp_layer_norm(self, X, T, gain=None, bias=None, eps=1e-5, out=None):
        """Normalisation of every token over the channels of X [d x ld]; gain, bias [d] fp32.  out may be X."""
        d = X.shape[0]
        if out is None:
            out = self._new(d, T, X.dtype)
        ldx, ldy = self._matrix("X", X, d, T, _CODES), self._matrix("out", out, d, T, (X.dtype,))
        self.check(self.lib.strp_layer_norm(self.h, X.data_ptr(), _CODES[X.dtype], d, T, ldx, self._vector("gain", gain, d, torch.float32),
                                            self._vector("bias", bias, d, torch.float32), eps, out.data_ptr(), ldy))
        return out

    def strp_attention(self, Q, K, V, T, heads, kv_heads=None, seq_start=None, kv_of_head=None, scale=None, out=None):
        """Causal attention of T packed tokens: Q [heads*d_head x ld], K, V [kv_heads*d_head x ld], seq_start [n_seq + 1] int32 offsets
        (None: one sequence), kv_of_head [heads] int32 (None: equal groups), scale 1 / sqrt(d_head) by default.  In bf16 the
        probabilities are held in two terms, or rounded once where the context's precision is PREC_FAST.  Returns the head outputs, like Q."""
        kv_heads = heads if kv_heads is None else kv_heads
        if heads <= 0 or Q.dim() != 2 or Q.shape[0] < heads or Q.shape[0] % heads:
            raise ValueError(f"Q: {tuple(Q.shape)} is not {heads} heads")
        rows, same = Q.shape[0], (Q.dtype,)
        dh = rows // heads
        if out is None:
            out = self._new(rows, T, Q.dtype)
        ldq, ldk = self._matrix("Q", Q, rows, T, _CODES), self._matrix("K", K, kv_heads * dh, T, same)
        ldv, ldc = self._matrix("V", V, kv_heads * dh, T, same), self._matrix("out", out, rows, T, same)
        n_seq = 0 if seq_start is None else seq_start.shape[0] - 1
        self.check(self.lib.strp_attention(self.h, _ATTENTION.pack(
            Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), self._vector("seq_start", seq_start, 2, torch.int32),
            self._vector("kv_of_head", kv_of_head, heads, torch.int32), _CODES[Q.dtype], heads, kv_heads, dh, n_seq,
            dh ** -0.5 if scale is None else scale, T, ldq, ldk, ldv, ldc)))
        return out

    def strp_token_logprobs(self, logits, T, target=None, entropy=True, n_top=0):
        """What a model answers at each of T tokens, from logits [V x ld]: dict of logp [T] (of target [T] int32, if given), entropy [T]
        (if wanted), top_ids and top_logp [n_top x T]."""
        V = logits.shape[0]
        ldl = self._matrix("logits", logits, V, T, _CODES)
        y = self._vector("target", target, T, torch.int32)
        if n_top < 0 or n_top > min(V, TOP_MAX):
            raise ValueError(f"n_top outside [0, {min(V, TOP_MAX)}]")
        if T <= 0:
            raise ValueError(f"{T} tokens")
        # one allocation for what is fp32
        rows = (target is not None) + bool(entropy) + n_top
        floats = self._empty((rows, T), torch.float32)
        res, at = {}, 0
        if target is not None:
            res["logp"], at = floats[0], 1
        if entropy:
            res["entropy"], at = floats[at], at + 1
        res["top_ids"], res["top_logp"] = self._empty((n_top, T), torch.int32), floats[at:]
        self.ensure_workspace(self.lib.strp_token_logprobs_workspace_bytes(V, T, n_top))
        base, row = floats.data_ptr(), 4 * T
        self.check(self.lib.strp_token_logprobs(self.h, logits.data_ptr(), _CODES[logits.dtype], V, T, ldl, y or None, base if y else None,
                                                base + (row if y else 0) if entropy else None, n_top, res["top_ids"].data_ptr() if n_top else None,
                                                base + at * row if n_top else None, T))
        return res

    # ---- what a model needs to generate ---------------------------------------------------
    def _pages(self, cache, table, past, seq_start, T):
        """Fields of strp_cache for a call on T tokens."""
        if cache.device != self.index or table.get_device() != self.index:
            raise ValueError(f"the cache or its table is not on {self.device}")
        if table.dtype is not torch.int32 or table.dim() != 2 or not table.is_contiguous():
            raise ValueError("table: needs contiguous int32 rows, one a sequence")
        n_seq, ld = table.shape
        return cache.fields[:4] + (table.data_ptr(), self._vector("past", past, n_seq, torch.int32), self._vector("seq_start", seq_start, n_seq + 1, torch.int32)) + cache.fields[4:] + (n_seq, ld)

    def strp_cache_append(self, K, V, T, cache, table, past, seq_start=None, inv_freq=None, pairs=False, Q=None, q_out=None):
        """Keys and values [kv_heads*d_head x ld] of T new tokens into the cache's pages: those of sequence i (tokens seq_start[i] to seq_start[i + 1]; None:
        one sequence of all) behind the past[i] that it has, in the pages table[i].  inv_freq [rot / 2] fp32: the first rot channels of every head of K and Q are
        turned by position * inv_freq, channels (j, j + rot / 2) together, or (2j, 2j + 1) with pairs.  Returns Q turned (q_out may be Q), None without Q."""
        dt, dh = K.dtype, cache.d_head
        rows = cache.kv_heads * dh
        ldk, ldv = self._matrix("K", K, rows, T, _CODES), self._matrix("V", V, rows, T, (dt,))
        heads = q = r = ldq = ldr = 0
        if Q is not None:
            if Q.dim() != 2 or Q.shape[0] % dh:
                raise ValueError(f"Q: {tuple(Q.shape)} is not heads of {dh}")
            rows = Q.shape[0]
            heads = rows // dh
            ldq = self._matrix("Q", Q, rows, T, (dt,))
            if q_out is None:
                q_out = self._new(rows, T, dt)
            ldr = ldq if q_out is Q else self._matrix("q_out", q_out, rows, T, (dt,))
            q, r = Q.data_ptr(), q_out.data_ptr()
        rot = 0 if inv_freq is None else 2 * inv_freq.shape[0]
        self.check(self.lib.strp_cache_append(self.h, _CACHE_APPEND.pack(
            *self._pages(cache, table, past, seq_start, T), K.data_ptr(), V.data_ptr(), q, r, self._vector("inv_freq", inv_freq, rot // 2, torch.float32),
            _CODES[dt], heads, rot, bool(pairs), T, ldk, ldv, ldq, ldr)))
        return q_out if q else None

    def strp_cache_attention(self, Q, T, heads, cache, table, past, seq_start=None, kv_of_head=None, scale=None, out=None):
        """Attention of T new tokens over the cache, which holds them already (strp_cache_append with the same table, past and seq_start): a token sees its
        sequence up to itself.  Q [heads*d_head x ld], kv_of_head [heads] int32 (None: equal groups), scale 1 / sqrt(d_head) by default.  Returns the
        head outputs, like Q."""
        dh = cache.d_head
        ldq = self._matrix("Q", Q, heads * dh, T, _CODES)
        if out is None:
            out = self._new(heads * dh, T, Q.dtype)
        ldc = self._matrix("out", out, heads * dh, T, (Q.dtype,))
        self.ensure_workspace(self.lib.strp_cache_attention_workspace_bytes(dh))
        self.check(self.lib.strp_cache_attention(self.h, _CACHE_ATTENTION.pack(
            *self._pages(cache, table, past, seq_start, T), Q.data_ptr(), out.data_ptr(), self._vector("kv_of_head", kv_of_head, heads, torch.int32),
            _CODES[Q.dtype], heads, dh ** -0.5 if scale is None else scale, T, ldq, ldc)))
        return out

    def strp_verify_draft(self, target, draft, draft_ids, u, u_next, seq_start=None, temperature=1.0):
        """Which drafted tokens the target keeps, and the token that follows: dict of accepted and next_ids [n_seq] int32.  target [V x ld] logits at every
        drafted position and behind the last one of each sequence, draft [V x ld] at the drafted positions, draft_ids [T] int32, u [T] and u_next
        [n_seq] fp32 random numbers in [0, 1), seq_start [n_seq + 1] int32 (None: one sequence).  draft, draft_ids and u None: one token of
        each sequence is sampled from the target."""
        n_seq = u_next.shape[0]
        T = 0 if draft is None else draft_ids.shape[0]
        V = target.shape[0]
        ldt = self._matrix("target", target, V, T + n_seq, _CODES)
        d = ids = uu = ldd = 0
        if T:
            ldd = self._matrix("draft", draft, V, T, (target.dtype,))
            d, ids, uu = draft.data_ptr(), self._vector("draft_ids", draft_ids, T, torch.int32), self._vector("u", u, T, torch.float32)
        elif draft_ids is not None and draft_ids.shape[0]:
            raise ValueError("draft_ids without draft")
        starts = self._vector("seq_start", seq_start, n_seq + 1, torch.int32)
        res = self._empty((2, n_seq), torch.int32)
        self.ensure_workspace(self.lib.strp_verify_draft_workspace_bytes(V, T, n_seq))
        self.check(self.lib.strp_verify_draft(self.h, _VERIFY_DRAFT.pack(
            target.data_ptr(), d, ids, uu, self._vector("u_next", u_next, n_seq, torch.float32), starts, res.data_ptr(), res.data_ptr() + 4 * n_seq,
            _CODES[target.dtype], V, n_seq, float(temperature), T, ldt, ldd)))
        return dict(accepted=res[0], next_ids=res[1])

    def strp_module_init(self, desc, state, params):
        self.check(self.lib.strp_module_init(self.h, C.byref(desc), C.byref(state), C.byref(params)))

    def strp_admm_step(self, desc, state, params, report=True):
        rep = Report() if report else None
        self.check(self.lib.strp_admm_step(self.h, C.byref(desc), C.byref(state), C.byref(params),
                                           C.byref(rep) if rep is not None else None))
        return rep


class PagedCache:
    """Pages of keys and values: K, V [pages x kv_heads x page x d_head] of bf16 or fp32, or uint8 [.. x d_head / 2] for 4 bits, then with
    K_scale, V_scale [pages x kv_heads x page x 2] fp32 (lowest, step).  A program keeps one for a layer and hands pages to sequences as it likes."""

    def __init__(self, K, V, K_scale=None, V_scale=None):
        q4 = K.dtype is torch.uint8
        scales = (K_scale, V_scale) if q4 else ()
        if K.dtype not in (torch.bfloat16, torch.float32, torch.uint8) or K.dim() != 4 or V.dtype is not K.dtype or V.shape != K.shape:
            raise ValueError("K and V: [pages x kv_heads x page x d_head], both bf16, fp32, or uint8 (4 bits)")
        if not q4 and (K_scale is not None or V_scale is not None):
            raise ValueError("K_scale and V_scale belong to a cache of 4 bits")
        if any(t is None or t.dtype is not torch.float32 or t.shape != K.shape[:3] + (2,) for t in scales):
            raise ValueError("a cache of 4 bits needs K_scale and V_scale [pages x kv_heads x page x 2] fp32")
        if any(not t.is_contiguous() or t.get_device() != K.get_device() for t in (K, V) + scales):
            raise ValueError("the cache's tensors must be contiguous and on one device")
        self.K, self.V, self.K_scale, self.V_scale = K, V, K_scale, V_scale
        pages, self.kv_heads, self.page, width = K.shape
        self.d_head, self.device = width * (2 if q4 else 1), K.get_device()
        # as strp_cache has them, round what a call adds
        self.fields = (K.data_ptr(), V.data_ptr()) + (tuple(t.data_ptr() for t in scales) or (0, 0)) + (CACHE_Q4 if q4 else _CODES[K.dtype], self.kv_heads, self.d_head, self.page, pages)

    @classmethod
    def empty(cls, ctx, pages, kv_heads, d_head, page=64, dtype=torch.bfloat16):
        """A cache of `dtype` (torch.uint8: 4 bits) with nothing in it."""
        with torch.cuda.stream(ctx.stream):
            e = lambda width, dt: torch.empty((pages, kv_heads, page, width), dtype=dt, device=ctx.device)
            if dtype is torch.uint8:
                return cls(e(d_head // 2, dtype), e(d_head // 2, dtype), e(2, torch.float32), e(2, torch.float32))
            return cls(e(d_head, dtype), e(d_head, dtype))


class FFNModule:
    """Device buffers of one resident FFN module plus the ctypes structs that describe them."""

    def __init__(self, ctx: Context, W1hat: torch.Tensor, W2hat: torch.Tensor, X: torch.Tensor, T: int,
                 k_max: int = 0):
        dev = ctx.device
        f, d = W1hat.shape
        self.ctx, self.d, self.f, self.T = ctx, d, f, T
        self.W1hat, self.W2hat, self.X = W1hat.contiguous(), W2hat.contiguous(), X
        lda = (T + 7) // 8 * 8
        self.lda = lda
        e = lambda *shape, dt=torch.float32: torch.empty(shape, dtype=dt, device=dev)
        self.Z, self.A, self.Z0 = e(f, lda), e(f, lda), e(f, lda)
        self.Y = e(d, lda)
        self.W1, self.W2 = e(f, d), e(d, f)
        self.H = e(d, d)
        self.cholH = e(d, d, dt=torch.float64)
        self.n2 = e(f, dt=torch.float64)
        self.score = e(f)
        self.mask = e(f, dt=torch.uint8)
        self.idx = e(f, dt=torch.int32)
        self.scalars = torch.zeros(32, dtype=torch.float64, device=dev)
        self.desc = ModuleDesc(d, f, T, X.stride(0), lda, dtype_code(X), dtype_code(W1hat), k_max)
        self.cache = torch.empty(int(ctx.lib.strp_module_cache_bytes(C.byref(self.desc))), dtype=torch.uint8, device=dev)
        st = ModuleState()
        for name in ("X", "W1hat", "W2hat", "Z", "A", "Z0", "Y", "W1", "W2", "H", "cholH", "n2", "score", "mask",
                     "idx", "scalars", "cache"):
            setattr(st, name, getattr(self, name).data_ptr())
        st.s, st.iter = 0, 0
        self.state = st
        ctx.ensure_workspace(ctx.workspace_bytes(self.desc))

    def rebind_inputs(self, W1hat: torch.Tensor, W2hat: torch.Tensor, X: torch.Tensor):
        """Point the state at another module's inputs of the same shapes (the state buffers are reused; call init next)."""
        assert W1hat.shape == self.W1hat.shape and W2hat.shape == self.W2hat.shape and X.shape == self.X.shape
        assert W1hat.dtype == self.W1hat.dtype and X.dtype == self.X.dtype and X.stride(0) == self.X.stride(0)
        self.W1hat, self.W2hat, self.X = W1hat, W2hat, X
        for name in ("X", "W1hat", "W2hat"):
            setattr(self.state, name, getattr(self, name).data_ptr())

    def init(self, params: Params):
        self.ctx.strp_module_init(self.desc, self.state, params)

    def step(self, params: Params, report=True):
        return self.ctx.strp_admm_step(self.desc, self.state, params, report)

    @property
    def s(self):
        return int(self.state.s)
