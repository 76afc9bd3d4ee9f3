"""Thin ctypes binding of libscd.so (the C ABI in include/scd.h).

Argument marshalling only: every step of the decode iteration runs in the HIP
kernels.  PyTorch is used for device memory and the current HIP stream.  The
functions carry the same names as the C entry points.  There is no CPU
fallback: if the shared library is missing, loading raises.
"""
import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libscd.so")

SCD_OK, SCD_EINVAL, SCD_EWORKSPACE, SCD_EHIP, SCD_ENUMERIC, SCD_EUNSUPPORTED, SCD_ESCRATCH = 0, -1, -2, -3, -4, -5, -6
STATIC_SCRATCH_BYTES = 8 << 20

# scd_field
(F_POS, F_ITER, F_X, F_AGE, F_OUT, F_ACCEPT, F_Y, F_K, F_PX, F_QX, F_THR, F_LSE, F_NKEPT, F_Z,
 F_FLAGS, F_VERIFIED, F_TICKET, F_G, F_DIAG, F_S2, F_HAMM, F_XHIST, F_PHIST) = range(23)
F_COUNT = 23
COUPLING_MC, COUPLING_GS = 0, 1

_FIELD_DTYPE = {
    F_POS: torch.int32, F_ITER: torch.int32, F_X: torch.int32, F_AGE: torch.int32,
    F_OUT: torch.int32, F_ACCEPT: torch.int32, F_Y: torch.int32, F_K: torch.uint8,
    F_PX: torch.float32, F_QX: torch.float32, F_THR: torch.float32, F_LSE: torch.float32,
    F_NKEPT: torch.int32, F_Z: torch.float32, F_FLAGS: torch.int32, F_VERIFIED: torch.int32,
    F_TICKET: torch.int32, F_G: torch.int32, F_DIAG: torch.float32, F_S2: torch.float32,
    F_HAMM: torch.int32, F_XHIST: torch.int32, F_PHIST: torch.int32,
}


class ScdConfig(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("L", ctypes.c_int32), ("N", ctypes.c_int32),
                ("V", ctypes.c_int32), ("d", ctypes.c_int32), ("v_lo", ctypes.c_int32),
                ("v_hi", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("cfg_lambda", ctypes.c_float),
                ("coupling", ctypes.c_int32), ("sjd_mix", ctypes.c_float),
                ("top_p", ctypes.c_float), ("diagnostics", ctypes.c_int32),
                ("seed", ctypes.c_uint64)]


class ScdQuantized(ctypes.Structure):
    _fields_ = [("d_packed", ctypes.c_void_p), ("group", ctypes.c_int32), ("zeros", ctypes.c_int32)]


class ScdTensor(ctypes.Structure):
    _fields_ = [("d", ctypes.c_void_p), ("n", ctypes.c_int64), ("type", ctypes.c_int32)]


class ScdError(RuntimeError):
    def __init__(self, code, what):
        super().__init__(f"{what}: {code} ({strerror(code)})")
        self.code = code


_lib = None


def load():
    """Loads libscd.so (built in-tree by paper_2510_24211_amd.build).  Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    path = os.environ.get("SCD_LIB", LIB_PATH)      # SCD_LIB: an alternative build of the library
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with "
                           "`python -m paper_2510_24211_amd.build` (there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    cfgp = ctypes.POINTER(ScdConfig)
    lib.scd_workspace_bytes.restype = sz
    lib.scd_workspace_bytes.argtypes = [cfgp]
    lib.scd_state_bytes.restype = sz
    lib.scd_state_bytes.argtypes = [cfgp]
    lib.scd_create.argtypes = [ctypes.POINTER(vp), cfgp, vp, sz, vp]
    lib.scd_destroy.argtypes = [vp]
    lib.scd_reset.argtypes = [vp, vp]
    lib.scd_state_field.argtypes = [vp, vp, ctypes.c_int, ctypes.POINTER(vp), ctypes.POINTER(sz)]
    lib.scd_lm_head.argtypes = [vp, vp, vp, vp]
    lib.scd_select.argtypes = [vp, vp, i32, vp, vp, vp]
    lib.scd_couple_draft.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.scd_couple_draft_static.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.scd_verify.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.scd_step.argtypes = [vp, vp, vp, vp]
    lib.scd_step_logits.argtypes = [vp, vp, vp]
    lib.scd_set_lm_head_events.argtypes = [vp, vp, vp]
    lib.scd_lm_head_kernel_name.argtypes = [vp, ctypes.c_char_p, sz]
    f32 = ctypes.c_float
    quantp = ctypes.POINTER(ScdQuantized)
    lib.scd_quantized_bytes.restype = sz
    lib.scd_quantized_bytes.argtypes = [cfgp, i32, i32]
    lib.scd_quantize.argtypes = [vp, vp, i32, vp, vp, vp]
    lib.scd_pack_quantized.argtypes = [vp, vp, vp, vp, i32, vp]
    lib.scd_lm_head_quantized.argtypes = [vp, vp, quantp, vp]
    lib.scd_step_quantized.argtypes = [vp, vp, quantp, vp]
    lib.scd_lm_head_quantized_kernel_name.argtypes = [vp, i32, i32, ctypes.c_char_p, sz]
    lib.scd_embed.argtypes = [vp, vp, i32, vp, f32, vp]
    lib.scd_embed_window.argtypes = [vp, vp, vp, f32, vp]
    lib.scd_embed_backward_workspace_bytes.restype = sz
    lib.scd_embed_backward_workspace_bytes.argtypes = [cfgp, i32]
    lib.scd_embed_backward.argtypes = [vp, vp, i32, vp, f32, vp, i32, i32, vp, sz]
    lib.scd_cross_entropy_workspace_bytes.restype = sz
    lib.scd_cross_entropy_workspace_bytes.argtypes = [cfgp, i32]
    lib.scd_cross_entropy.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, sz]
    lib.scd_cross_entropy_backward_workspace_bytes.restype = sz
    lib.scd_cross_entropy_backward_workspace_bytes.argtypes = [cfgp, i32, i32]
    lib.scd_cross_entropy_backward.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, i32, vp, sz]
    lib.scd_cross_entropy_kernel_names.argtypes = [vp, i32, i32, ctypes.c_char_p, sz]
    tensorp = ctypes.POINTER(ScdTensor)
    lib.scd_norm.argtypes = [vp, vp, vp, i32, vp, i32, f32, i32, vp, vp, vp]
    lib.scd_norm_fp8.argtypes = [vp, vp, vp, i32, vp, i32, f32, i32, vp, vp, vp, vp]
    lib.scd_norm_backward_workspace_bytes.restype = sz
    lib.scd_norm_backward_workspace_bytes.argtypes = [cfgp, i32]
    lib.scd_norm_backward.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp, i32, i32, vp, vp, i32, i32, vp, sz]
    lib.scd_quantize_fp8.argtypes = [vp, vp, vp, vp]
    lib.scd_lm_head_fp8.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.scd_step_fp8.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.scd_lm_head_fp8_kernel_name.argtypes = [vp, ctypes.c_char_p, sz]
    lib.scd_gradient_norm_workspace_bytes.restype = sz
    lib.scd_gradient_norm_workspace_bytes.argtypes = [tensorp, i32]
    lib.scd_gradient_norm.argtypes = [vp, tensorp, i32, vp, vp, sz]
    lib.scd_clip_gradients.argtypes = [vp, tensorp, tensorp, i32, f32, vp]
    lib.scd_status.argtypes = [vp, vp, ctypes.POINTER(i32 * 4)]
    lib.scd_strerror.restype = ctypes.c_char_p
    lib.scd_strerror.argtypes = [ctypes.c_int]
    lib.scdw_gather_hidden.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.scdw_copy.argtypes = [vp, vp, vp, sz]
    for name in ("scd_create", "scd_destroy", "scd_reset", "scd_state_field", "scd_lm_head",
                 "scd_select", "scd_couple_draft", "scd_couple_draft_static", "scd_verify", "scd_step", "scd_step_logits",
                 "scd_set_lm_head_events", "scd_lm_head_kernel_name", "scd_quantize",
                 "scd_pack_quantized", "scd_lm_head_quantized", "scd_step_quantized", "scd_lm_head_quantized_kernel_name", "scd_embed", "scd_embed_window",
                 "scd_embed_backward", "scd_cross_entropy", "scd_cross_entropy_backward",
                 "scd_cross_entropy_kernel_names", "scd_norm", "scd_norm_fp8", "scd_norm_backward", "scd_quantize_fp8",
                 "scd_lm_head_fp8", "scd_step_fp8", "scd_lm_head_fp8_kernel_name", "scd_gradient_norm", "scd_clip_gradients", "scd_status", "scdw_gather_hidden", "scdw_copy"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def strerror(code):
    return load().scd_strerror(int(code)).decode()


def make_config(B, L, N, V, d=0, v_lo=0, v_hi=-1, top_k=0, temperature=1.0, cfg_lambda=0.0,
                seed=0, coupling=0, sjd_mix=0.0, top_p=0.0, diagnostics=0):
    return ScdConfig(B, L, N, V, d, v_lo, V if v_hi < 0 else v_hi, top_k, temperature, cfg_lambda,
                     coupling, sjd_mix, top_p, diagnostics, seed & 0xFFFFFFFFFFFFFFFF)


def workspace_bytes(cfg):
    return load().scd_workspace_bytes(ctypes.byref(cfg))


def state_bytes(cfg):
    return load().scd_state_bytes(ctypes.byref(cfg))


def _ptr(t, dtypes, numel, what):
    """Device address of a contiguous CUDA tensor after checking dtype and size."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{what}: dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: tensor must be contiguous")
    if t.numel() < numel:
        raise ValueError(f"{what}: {t.numel()} elements, need {numel}")
    return t.data_ptr()


def _int32(value, what):
    """`value` for an int32 argument: ctypes cuts off what does not fit."""
    value = int(value)
    if not -(1 << 31) <= value < 1 << 31:
        raise ValueError(f"{what}: {value} does not fit 32 bits")
    return value


_BF16 = (torch.bfloat16, torch.int16, torch.uint16)
GRAD_BF16, GRAD_F32 = 0, 1
_GRAD = {torch.bfloat16: GRAD_BF16, torch.float32: GRAD_F32}


def _grad_type(dtype):
    if dtype not in _GRAD:
        raise TypeError(f"gradient of W: dtype {dtype}, expected one of {tuple(_GRAD)}")
    return _GRAD[dtype]


_E4M3 = (torch.float8_e4m3fn, torch.uint8)
_F32 = (torch.float32,)
BF16, F32 = 0, 1
_TYPE = {torch.bfloat16: BF16, torch.float32: F32}


_TYPES = tuple(_TYPE)


def _typed(t, numel, what):
    """Device address and scd_type of a tensor; of none, any."""
    p = _ptr(t, _TYPES, numel, what)
    return p, BF16 if t is None else _TYPE[t.dtype]


class TensorList:
    """Tensors (contiguous, bf16 or fp32, views among them) as gradient_norm and clip_gradients take them: the memory that they have now, which
    the list keeps alive.  A tensor that has other memory later (its data exchanged, its storage resized) needs a new list: calls refuse this one."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.array = (ScdTensor * max(1, len(self.tensors)))()
        for i, t in enumerate(self.tensors):
            p = _ptr(t, _TYPES, 0, f"tensor {i}")
            if p is None:
                raise TypeError(f"tensor {i}: expected a CUDA tensor")
            self.array[i] = ScdTensor(p, t.numel(), _TYPE[t.dtype])
        self._memory = [t.detach() for t in self.tensors]
        self._addresses = [t.data_ptr() for t in self.tensors]

    def __len__(self):
        return len(self.tensors)

    def check(self, what):
        """Raises ValueError if a tensor's memory is not the one it had."""
        now = [t.data_ptr() for t in self.tensors]
        if now != self._addresses:
            i = next(i for i, (a, b) in enumerate(zip(now, self._addresses)) if a != b)
            raise ValueError(f"{what}: tensor {i} has other memory than when the list was made")


class QuantizedWeights:
    """4-bit weights as pack_quantized lays them out for one configuration's allowed ids and width; cfg = None: the
    caller answers for that."""

    def __init__(self, data, group, zeros, cfg=None):
        self.data, self.group, self.zeros = data, group, zeros
        self.rows = None if cfg is None else (cfg.v_lo, cfg.v_hi, cfg.d)


class Scd:
    """One scd_ctx plus its workspace.  Methods = the C entry points."""

    def __init__(self, cfg: ScdConfig, device="cuda:0", stream=None):
        self.lib = load()
        self.cfg = cfg
        self.device = torch.device(device)
        self.n = cfg.v_hi - cfg.v_lo
        self.C = 2 if cfg.cfg_lambda != 0.0 else 1
        need = self.lib.scd_workspace_bytes(ctypes.byref(cfg))
        if need == 0:
            raise ScdError(SCD_EINVAL, "scd_workspace_bytes")
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.workspace = self._empty(need)
        ctx = ctypes.c_void_p()
        rc = self.lib.scd_create(ctypes.byref(ctx), ctypes.byref(cfg),
                                 ctypes.c_void_p(self.workspace.data_ptr()), need,
                                 ctypes.c_void_p(self.stream.cuda_stream))
        if rc != SCD_OK:
            raise ScdError(rc, "scd_create")
        self.ctx = ctx

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.scd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        self.close()

    @staticmethod
    def _check(rc, what):
        if rc != SCD_OK:
            raise ScdError(rc, what)

    def _empty(self, nbytes):
        """Memory of the context's stream: what another stream has freed may be in use there still."""
        if torch.cuda.current_stream(self.device) == self.stream:
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    # -- state ------------------------------------------------------------
    def alloc_state(self):
        return self._empty(self.lib.scd_state_bytes(ctypes.byref(self.cfg)))

    def state_field(self, state, field):
        """A tensor view of one field of the state buffer."""
        p, nb = ctypes.c_void_p(), ctypes.c_size_t()
        self._check(self.lib.scd_state_field(self.ctx, ctypes.c_void_p(state.data_ptr()), field,
                                             ctypes.byref(p), ctypes.byref(nb)), "scd_state_field")
        off = p.value - state.data_ptr()
        return state[off: off + nb.value].view(_FIELD_DTYPE[field])

    def reset(self, state):
        self._check(self.lib.scd_reset(self.ctx, _ptr(state, (torch.uint8,),
                                                      state_bytes(self.cfg), "state")), "scd_reset")

    def status(self, state):
        flags = (ctypes.c_int32 * 4)()
        rc = self.lib.scd_status(self.ctx, ctypes.c_void_p(state.data_ptr()), ctypes.byref(flags))
        return rc, list(flags)

    # -- stages -------------------------------------------------------------
    def lm_head(self, h, W, z):
        c = self.cfg
        self._check(self.lib.scd_lm_head(
            self.ctx, _ptr(h, _BF16, c.B * self.C * c.L * c.d, "h"),
            _ptr(W, _BF16, c.V * c.d, "W"),
            _ptr(z, (torch.float32,), c.B * c.L * self.n, "z")), "scd_lm_head")

    def select(self, z, rows, thr, lse, nkept):
        self._check(self.lib.scd_select(
            self.ctx, _ptr(z, (torch.float32,), rows * self.n, "z"), rows,
            _ptr(thr, (torch.float32,), rows, "thr"), _ptr(lse, (torch.float32,), rows, "lse"),
            _ptr(nkept, (torch.int32,), rows, "nkept")), "scd_select")

    def couple_draft_static(self, z_cur, z_prev, x, fresh, pos0, it, y, k):
        """scd_couple_draft with its scratch in the library's static device array."""
        c = self.cfg
        r = c.B * c.L
        self._check(self.lib.scd_couple_draft_static(
            self.ctx, _ptr(z_cur, (torch.float32,), r * self.n, "z_cur"),
            _ptr(z_prev, (torch.float32,), r * self.n, "z_prev"),
            _ptr(x, (torch.int32,), r, "x"), _ptr(fresh, (torch.uint8,), r, "fresh"),
            _ptr(pos0, (torch.int32,), c.B, "pos0"), int(it),
            _ptr(y, (torch.int32,), r, "y"), _ptr(k, (torch.uint8,), r, "k")), "scd_couple_draft_static")

    def couple_draft(self, z_cur, z_prev, x, fresh, pos0, it, y, k):
        c = self.cfg
        r = c.B * c.L
        self._check(self.lib.scd_couple_draft(
            self.ctx, _ptr(z_cur, (torch.float32,), r * self.n, "z_cur"),
            _ptr(z_prev, (torch.float32,), r * self.n, "z_prev"),
            _ptr(x, (torch.int32,), r, "x"), _ptr(fresh, (torch.uint8,), r, "fresh"),
            _ptr(pos0, (torch.int32,), c.B, "pos0"), int(it),
            _ptr(y, (torch.int32,), r, "y"), _ptr(k, (torch.uint8,), r, "k")), "scd_couple_draft")

    def verify(self, k, y, pos0, accept_len, out):
        c = self.cfg
        r = c.B * c.L
        self._check(self.lib.scd_verify(
            self.ctx, _ptr(k, (torch.uint8,), r, "k"), _ptr(y, (torch.int32,), r, "y"),
            _ptr(pos0, (torch.int32,), c.B, "pos0"),
            _ptr(accept_len, (torch.int32,), c.B, "accept_len"),
            _ptr(out, (torch.int32,), c.B * c.N, "out")), "scd_verify")

    def step(self, h, W, state):
        c = self.cfg
        self._check(self.lib.scd_step(
            self.ctx, _ptr(h, _BF16, c.B * self.C * c.L * c.d, "h"),
            _ptr(W, _BF16, c.V * c.d, "W"),
            _ptr(state, (torch.uint8,), state_bytes(c), "state")), "scd_step")

    def set_lm_head_events(self, ev_start, ev_stop):
        """ev_*: hipEvent_t handles as integers (or None, None to turn off)."""
        self._check(self.lib.scd_set_lm_head_events(
            self.ctx, ctypes.c_void_p(ev_start) if ev_start else None,
            ctypes.c_void_p(ev_stop) if ev_stop else None), "scd_set_lm_head_events")

    def lm_head_kernel_name(self):
        buf = ctypes.create_string_buffer(96)
        self._check(self.lib.scd_lm_head_kernel_name(self.ctx, buf, 96), "scd_lm_head_kernel_name")
        return buf.value.decode()

    def step_logits(self, z, state):
        c = self.cfg
        self._check(self.lib.scd_step_logits(
            self.ctx, _ptr(z, (torch.float32,), c.B * c.L * self.n, "z"),
            _ptr(state, (torch.uint8,), state_bytes(c), "state")), "scd_step_logits")

    # -- 4-bit weights ----------------------------------------------------------
    def quantize(self, W, group, codes, scales, zeros=None):
        c, group = self.cfg, _int32(group, "group")
        G = -(-c.d // group) if group > 0 else 0
        self._check(self.lib.scd_quantize(
            self.ctx, _ptr(W, _BF16, c.V * c.d, "W"), group, _ptr(codes, (torch.uint8,), c.V * c.d // 2, "codes"),
            _ptr(scales, _BF16, c.V * G, "scales"), _ptr(zeros, (torch.uint8,), c.V * G, "zeros")), "scd_quantize")

    def pack_quantized(self, codes, scales, zeros, group):
        """The weights in the layout that lm_head_quantized and step_quantized read, in memory of their own."""
        c, group = self.cfg, _int32(group, "group")
        need = self.lib.scd_quantized_bytes(ctypes.byref(c), group, int(zeros is not None))
        G = -(-c.d // group) if need else 0
        packed = QuantizedWeights(self._workspace(need, "scd_quantized_bytes"), group, zeros is not None, c)
        self._check(self.lib.scd_pack_quantized(
            self.ctx, _ptr(codes, (torch.uint8,), c.V * c.d // 2, "codes"), _ptr(scales, _BF16, c.V * G, "scales"),
            _ptr(zeros, (torch.uint8,), c.V * G, "zeros"), group, ctypes.c_void_p(packed.data.data_ptr())), "scd_pack_quantized")
        return packed

    def _quantized(self, W):
        group, rows = _int32(W.group, "group"), (self.cfg.v_lo, self.cfg.v_hi, self.cfg.d)
        if W.rows not in (None, rows):
            raise ValueError(f"quantized weights: laid out for (v_lo, v_hi, d) = {W.rows}, not for {rows}")
        need = self.lib.scd_quantized_bytes(ctypes.byref(self.cfg), group, int(W.zeros))
        if need == 0:
            raise ScdError(SCD_EINVAL, "scd_quantized_bytes")
        return ctypes.byref(ScdQuantized(_ptr(W.data, (torch.uint8,), need, "quantized weights"), group, int(W.zeros)))

    def lm_head_quantized(self, h, W, z):
        c = self.cfg
        self._check(self.lib.scd_lm_head_quantized(
            self.ctx, _ptr(h, _BF16, c.B * self.C * c.L * c.d, "h"), self._quantized(W),
            _ptr(z, (torch.float32,), c.B * c.L * self.n, "z")), "scd_lm_head_quantized")

    def step_quantized(self, h, W, state):
        c = self.cfg
        self._check(self.lib.scd_step_quantized(
            self.ctx, _ptr(h, _BF16, c.B * self.C * c.L * c.d, "h"), self._quantized(W),
            _ptr(state, (torch.uint8,), state_bytes(c), "state")), "scd_step_quantized")

    def lm_head_quantized_kernel_name(self, group, zeros):
        buf = ctypes.create_string_buffer(128)
        self._check(self.lib.scd_lm_head_quantized_kernel_name(self.ctx, _int32(group, "group"), int(zeros), buf, 128),
                    "scd_lm_head_quantized_kernel_name")
        return buf.value.decode()

    # -- the vocabulary table at the model's other end, and what it learns ----------
    def _workspace(self, need, what):
        if need == 0:
            raise ScdError(SCD_EINVAL, what)
        return self._empty(need)

    def embed(self, ids, W, scale, x):
        """x[r] = scale * W[ids[r]] for every id of `ids`; zeros for ids outside [0, V)."""
        c, rows = self.cfg, _int32(ids.numel(), "ids")
        self._check(self.lib.scd_embed(
            self.ctx, _ptr(ids, (torch.int32,), rows, "ids"), rows, _ptr(W, _BF16, c.V * c.d, "W"), float(scale),
            _ptr(x, _BF16, rows * c.d, "x")), "scd_embed")

    def embed_window(self, state, W, scale, x):
        c = self.cfg
        self._check(self.lib.scd_embed_window(
            self.ctx, _ptr(state, (torch.uint8,), state_bytes(c), "state"), _ptr(W, _BF16, c.V * c.d, "W"), float(scale),
            _ptr(x, _BF16, c.B * self.C * c.L * c.d, "x")), "scd_embed_window")

    def embed_backward_workspace(self, rows):
        return self._workspace(self.lib.scd_embed_backward_workspace_bytes(ctypes.byref(self.cfg), _int32(rows, "rows")),
                               "scd_embed_backward_workspace_bytes")

    def embed_backward(self, ids, dx, scale, dW, workspace, accumulate=False):
        """dW (bf16 or fp32) = or += scale * the sums of dx's rows by id."""
        c, rows = self.cfg, _int32(ids.numel(), "ids")
        self._check(self.lib.scd_embed_backward(
            self.ctx, _ptr(ids, (torch.int32,), rows, "ids"), rows, _ptr(dx, _BF16, rows * c.d, "dx"), float(scale),
            _ptr(dW, tuple(_GRAD), c.V * c.d, "dW"), _grad_type(dW.dtype), int(accumulate),
            _ptr(workspace, (torch.uint8,), 1, "workspace"), workspace.numel()), "scd_embed_backward")

    def cross_entropy_workspace(self, rows):
        return self._workspace(self.lib.scd_cross_entropy_workspace_bytes(ctypes.byref(self.cfg), _int32(rows, "rows")),
                               "scd_cross_entropy_workspace_bytes")

    def cross_entropy(self, h, W, targets, loss, lse, workspace):
        """One loss and log normaliser per target; a negative target leaves its row out."""
        c, rows = self.cfg, _int32(targets.numel(), "targets")
        self._check(self.lib.scd_cross_entropy(
            self.ctx, _ptr(h, _BF16, rows * c.d, "h"), _ptr(W, _BF16, c.V * c.d, "W"),
            _ptr(targets, (torch.int32,), rows, "targets"), rows, _ptr(loss, (torch.float32,), rows, "loss"),
            _ptr(lse, (torch.float32,), rows, "lse"), _ptr(workspace, (torch.uint8,), 1, "workspace"),
            workspace.numel()), "scd_cross_entropy")

    def cross_entropy_backward_workspace(self, rows, grad_dtype=torch.bfloat16):
        return self._workspace(self.lib.scd_cross_entropy_backward_workspace_bytes(
            ctypes.byref(self.cfg), _int32(rows, "rows"), _grad_type(grad_dtype)), "scd_cross_entropy_backward_workspace_bytes")

    def cross_entropy_backward(self, h, W, targets, lse, weight, dh, dW, workspace, accumulate=False):
        """Gradients of sum(weight * loss) (weight None: 1); dh or dW may be None."""
        c, rows = self.cfg, _int32(targets.numel(), "targets")
        self._check(self.lib.scd_cross_entropy_backward(
            self.ctx, _ptr(h, _BF16, rows * c.d, "h"), _ptr(W, _BF16, c.V * c.d, "W"),
            _ptr(targets, (torch.int32,), rows, "targets"), rows, _ptr(lse, (torch.float32,), rows, "lse"),
            _ptr(weight, (torch.float32,), rows, "weight"), _ptr(dh, _BF16, rows * c.d, "dh"),
            _ptr(dW, tuple(_GRAD), c.V * c.d, "dW"), _grad_type(dW.dtype) if dW is not None else GRAD_BF16,
            int(accumulate), _ptr(workspace, (torch.uint8,), 1, "workspace"), workspace.numel()),
            "scd_cross_entropy_backward")

    def cross_entropy_kernel_names(self, rows, grad_dtype=torch.bfloat16):
        buf = ctypes.create_string_buffer(256)
        self._check(self.lib.scd_cross_entropy_kernel_names(self.ctx, _int32(rows, "rows"), _grad_type(grad_dtype), buf, 256),
                    "scd_cross_entropy_kernel_names")
        return buf.value.decode()

    # -- around the last norm, and what it leaves of the gradients ----------------
    def _rows(self, t, what):
        if not isinstance(t, torch.Tensor) or t.numel() % max(1, self.cfg.d):
            raise ValueError(f"{what}: expected a tensor of whole rows of {self.cfg.d}")
        return _int32(t.numel() // max(1, self.cfg.d), what)

    def _norm_args(self, x, gain, eps, residual, sum):
        """What both norms take alike, and the address of the stream behind the addition."""
        rows, d = self._rows(x, "x"), self.cfg.d
        n = rows * d
        if residual is not None and sum is not None and residual.dtype != sum.dtype:
            raise TypeError(f"sum: dtype {sum.dtype}, the residual's is {residual.dtype}")
        return rows, n, (self.ctx, _ptr(x, _BF16, n, "x"), *_typed(residual, n, "residual"), *_typed(gain, d, "gain"), float(eps), rows), _ptr(
            sum, _TYPES, n, "sum")

    def norm(self, x, gain, y, eps, residual=None, sum=None, inv=None):
        """y = s * inv * gain, s = x + residual (kept in sum, which may be residual), inv = 1 / sqrt(mean(s^2) + eps)."""
        rows, n, args, s = self._norm_args(x, gain, eps, residual, sum)
        self._check(self.lib.scd_norm(*args, _ptr(y, _BF16, n, "y"), s, _ptr(inv, _F32, rows, "inv")), "scd_norm")

    def norm_fp8(self, x, gain, codes, scales, eps, residual=None, sum=None, inv=None):
        """The same with y as e4m3 codes and a scale per 128 of a row."""
        rows, n, args, s = self._norm_args(x, gain, eps, residual, sum)
        self._check(self.lib.scd_norm_fp8(
            *args, _ptr(codes, _E4M3, n, "codes"), _ptr(scales, _F32, rows * -(-self.cfg.d // 128), "scales"), s, _ptr(inv, _F32, rows, "inv")),
            "scd_norm_fp8")

    def norm_backward_workspace(self, rows):
        return self._workspace(self.lib.scd_norm_backward_workspace_bytes(ctypes.byref(self.cfg), _int32(rows, "rows")),
                               "scd_norm_backward_workspace_bytes")

    def norm_backward(self, sum, gain, inv, dy, dx, dgain, workspace, dsum=None, accumulate=False):
        """dx (bf16 or fp32, as dsum): gradient of x and of the residual; dgain (bf16 or fp32, or None) = or += the gains'."""
        rows, d = self._rows(sum, "sum"), self.cfg.d
        n = rows * d
        if dsum is not None and dsum.dtype != dx.dtype:
            raise TypeError(f"dsum: dtype {dsum.dtype}, dx's is {dx.dtype}")
        dx, grad = _typed(dx, n, "dx")
        dgain, gain_grad = _typed(dgain, d, "dgain")
        self._check(self.lib.scd_norm_backward(
            self.ctx, *_typed(sum, n, "sum"), *_typed(gain, d, "gain"), _ptr(inv, _F32, rows, "inv"), _ptr(dy, _BF16, n, "dy"),
            _ptr(dsum, _TYPES, n, "dsum"), grad, rows, dx, dgain, gain_grad, int(accumulate), _ptr(workspace, (torch.uint8,), 1, "workspace"),
            workspace.numel()), "scd_norm_backward")

    def quantize_fp8(self, W, codes, scales):
        """W as e4m3 codes and a scale for each block of 128 x 128."""
        c = self.cfg
        G = -(-c.d // 128)
        self._check(self.lib.scd_quantize_fp8(
            self.ctx, _ptr(W, _BF16, c.V * c.d, "W"), _ptr(codes, _E4M3, c.V * c.d, "codes"),
            _ptr(scales, (torch.float32,), -(-c.V // 128) * G, "scales")), "scd_quantize_fp8")

    def _fp8(self, h, h_scales, W, W_scales):
        c = self.cfg
        rows, G = c.B * self.C * c.L, -(-c.d // 128)
        return (_ptr(h, _E4M3, rows * c.d, "h"), _ptr(h_scales, (torch.float32,), rows * G, "h_scales"), _ptr(W, _E4M3, c.V * c.d, "W"),
                _ptr(W_scales, (torch.float32,), -(-c.V // 128) * G, "W_scales"))

    def lm_head_fp8(self, h, h_scales, W, W_scales, z):
        self._check(self.lib.scd_lm_head_fp8(
            self.ctx, *self._fp8(h, h_scales, W, W_scales), _ptr(z, (torch.float32,), self.cfg.B * self.cfg.L * self.n, "z")), "scd_lm_head_fp8")

    def step_fp8(self, h, h_scales, W, W_scales, state):
        self._check(self.lib.scd_step_fp8(
            self.ctx, *self._fp8(h, h_scales, W, W_scales), _ptr(state, (torch.uint8,), state_bytes(self.cfg), "state")), "scd_step_fp8")

    def lm_head_fp8_kernel_name(self):
        buf = ctypes.create_string_buffer(128)
        self._check(self.lib.scd_lm_head_fp8_kernel_name(self.ctx, buf, 128), "scd_lm_head_fp8_kernel_name")
        return buf.value.decode()

    def gradient_norm_workspace(self, grads):
        return self._workspace(self.lib.scd_gradient_norm_workspace_bytes(grads.array, len(grads)), "scd_gradient_norm_workspace_bytes")

    def gradient_norm(self, grads, norm, workspace):
        """norm[0] = the 2-norm of all tensors of a TensorList together."""
        grads.check("grads")
        self._check(self.lib.scd_gradient_norm(
            self.ctx, grads.array, len(grads), _ptr(norm, (torch.float32,), 1, "norm"), _ptr(workspace, (torch.uint8,), 1, "workspace"),
            workspace.numel()), "scd_gradient_norm")

    def clip_gradients(self, grads, out, max_norm, norm):
        """out[i] = grads[i] * min(1, max_norm / norm[0]); out may be grads."""
        if len(grads) != len(out):
            raise ValueError(f"{len(out)} outputs for {len(grads)} tensors")
        grads.check("grads")
        out.check("out")
        self._check(self.lib.scd_clip_gradients(
            self.ctx, grads.array, out.array, len(grads), float(max_norm), _ptr(norm, (torch.float32,), 1, "norm")), "scd_clip_gradients")

    # -- benchmark plumbing ---------------------------------------------------
    def gather_hidden(self, table, age_cap, state, h):
        c = self.cfg
        rows = c.B * self.C * c.N * (age_cap + 1)
        rc = self.lib.scdw_gather_hidden(
            ctypes.c_void_p(self.stream.cuda_stream), _ptr(table, _BF16, rows * c.d, "table"),
            c.B, self.C, c.L, c.N, c.d, age_cap,
            ctypes.c_void_p(self.state_field(state, F_POS).data_ptr()),
            ctypes.c_void_p(self.state_field(state, F_AGE).data_ptr()),
            _ptr(h, _BF16, c.B * self.C * c.L * c.d, "h"))
        self._check(rc, "scdw_gather_hidden")


def device_copy(src, dst, stream=None):
    """dst <- src by the library's plain copy kernel (profiler counter calibration)."""
    assert src.is_cuda and dst.is_cuda and src.is_contiguous() and dst.is_contiguous()
    nbytes = src.numel() * src.element_size()
    assert nbytes == dst.numel() * dst.element_size()
    st = stream if stream is not None else torch.cuda.current_stream(src.device)
    rc = load().scdw_copy(ctypes.c_void_p(st.cuda_stream), ctypes.c_void_p(src.data_ptr()),
                          ctypes.c_void_p(dst.data_ptr()), nbytes)
    if rc != 0:
        raise RuntimeError(f"scdw_copy failed with {rc}")
    return nbytes


def config_from_workload(w):
    """ScdConfig for a paper_2510_24211_amd.workload.Workload."""
    return make_config(B=w.B, L=w.L, N=w.N, V=w.V, d=w.d, v_lo=w.v_lo, v_hi=w.v_hi, top_k=w.top_k,
                       temperature=w.temperature, cfg_lambda=w.cfg_lambda, seed=w.seed, top_p=w.top_p)
