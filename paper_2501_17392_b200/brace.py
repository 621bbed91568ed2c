"""ctypes binding of the BRACE CUDA library (C ABI in include/brace.h).

Argument marshalling only: every step of the aggregation runs in the CUDA
kernels.  torch is used for device memory and streams.  There is no CPU
fallback: if the compiled library is missing, loading raises.
"""

from __future__ import annotations

import ctypes as C
import os
import struct

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# BRACE_LIBRARY names another build of the same library (the debug build, for instance)
LIB_PATH = os.environ.get("BRACE_LIBRARY") or os.path.join(_PKG, "libbrace.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_BAD_STEP, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(7)
RULE_SIGN_CONSENSUS, RULE_SUM, RULE_MAJORITY_SIGN, RULE_ABS_CONSENSUS = 0, 1, 2, 3
AGG_AUTO, AGG_STEPWISE, AGG_FUSED = 0, 1, 2
STAT_MEDIAN, STAT_TRIMMED_MEAN = 0, 1
ATTACK_NONE, ATTACK_SCALE_OWN, ATTACK_GAUSSIAN, ATTACK_SCALED_MEAN, ATTACK_MEAN_SHIFT, ATTACK_SPARSE_NOISE = range(6)
DRAWS_SUPPLIED, DRAWS_GENERATED = 0, 1
DRAW_UNIFORM, DRAW_NORMAL = 0, 1
TYPE_F32, TYPE_BF16, TYPE_F16, TYPE_BITS = range(4)
ORTHO_AUTO, ORTHO_HALF, ORTHO_SINGLE = 0, 1, 2


class Params(C.Structure):
    _fields_ = [("rule", C.c_int32), ("lam", C.c_float), ("zero_sign", C.c_int32), ("granule", C.c_int32),
                ("mean", C.c_int32), ("agg_mode", C.c_int32)]


class Attack(C.Structure):
    _fields_ = [("kind", C.c_int32), ("scale", C.c_float), ("sigma", C.c_float), ("kappa", C.c_float),
                ("prob", C.c_float), ("h_byz_ids", C.POINTER(C.c_int32)), ("noise", C.c_void_p),
                ("noise_ld", C.c_int64), ("uniform", C.c_void_p), ("uniform_ld", C.c_int64),
                ("draws", C.c_int32), ("round", C.c_uint32), ("seed", C.c_uint64)]


class Cost(C.Structure):
    _fields_ = [("sc_bits", C.c_int64), ("rar_bits_min", C.c_int64), ("rar_bits_max", C.c_int64),
                ("brace_bits_min", C.c_int64), ("brace_bits_max", C.c_int64), ("packed_bits_min", C.c_int64),
                ("packed_bits_max", C.c_int64), ("rar_closed_form", C.c_double), ("brace_closed_form", C.c_double),
                ("partial_bits_used", C.c_int32), ("partial_bits_min", C.c_int32)]


class OrthoParams(C.Structure):
    _fields_ = [("steps", C.c_int32), ("a", C.c_float), ("b", C.c_float), ("c", C.c_float), ("eps", C.c_float),
                ("precision", C.c_int32)]


class Muon(C.Structure):
    _fields_ = [("d_grad", C.c_void_p), ("ld_grad", C.c_int64), ("stride_grad", C.c_int64),
                ("bit_offset", C.c_int64), ("d_momentum", C.c_void_p), ("ld_momentum", C.c_int64),
                ("stride_momentum", C.c_int64), ("d_momentum_out", C.c_void_p), ("ld_momentum_out", C.c_int64),
                ("stride_momentum_out", C.c_int64), ("d_weights", C.c_void_p), ("ld_weights", C.c_int64),
                ("stride_weights", C.c_int64), ("replica_weights", C.c_int64), ("d_weights_out", C.c_void_p),
                ("ld_weights_out", C.c_int64), ("stride_weights_out", C.c_int64),
                ("replica_weights_out", C.c_int64), ("grad_type", C.c_int32), ("weights_type", C.c_int32),
                ("replicas", C.c_int32), ("nesterov", C.c_int32), ("beta", C.c_float), ("lr", C.c_float),
                ("weight_decay", C.c_float), ("scale", C.c_float)]


class EmbeddingArgs(C.Structure):
    _fields_ = [("clients", C.c_int32), ("dim", C.c_int32), ("tokens", C.c_int64), ("vocab", C.c_int64),
                ("d_table", C.c_void_p), ("ld_table", C.c_int64), ("stride_table", C.c_int64), ("d_ids", C.c_void_p),
                ("stride_ids", C.c_int64), ("d_act", C.c_void_p), ("ld_act", C.c_int64), ("stride_act", C.c_int64),
                ("table_type", C.c_int32), ("act_type", C.c_int32), ("id_bytes", C.c_int32),
                ("accumulate", C.c_int32), ("scale", C.c_float)]


class BraceError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None

# name -> (restype, argtypes); one entry per function declared in include/brace.h
SIGNATURES = {
    "brace_status_string": (C.c_char_p, [C.c_int]),
    "brace_default_params": (C.c_int, [C.POINTER(Params)]),
    "brace_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int64, C.POINTER(Params)]),
    "brace_init": (C.c_int, [C.POINTER(C.c_void_p), C.c_int32, C.c_int32, C.c_int64, C.POINTER(Params), C.c_void_p,
                             C.c_size_t, C.c_void_p]),
    "brace_destroy": (C.c_int, [C.c_void_p]),
    "brace_segment": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
    "brace_last_cuda_error": (C.c_int, [C.c_void_p]),
    "brace_comm_cost": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(Cost)]),
    "brace_inject_attack": (C.c_int, [C.c_void_p, C.POINTER(Attack), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                      C.c_void_p]),
    "brace_draw_matrix": (C.c_int, [C.c_int32, C.c_uint64, C.c_uint32, C.c_int32, C.c_int32, C.c_int64, C.c_void_p,
                                    C.c_int64, C.c_float, C.c_float, C.c_void_p]),
    "brace_quantize": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]),
    "brace_ring_reduce_scatter_step": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]),
    "brace_consensus": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "brace_ring_allgather_step": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]),
    "brace_aggregate": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]),
    "brace_apply_update": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_float, C.c_void_p]),
    "brace_coordinate_stat": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p,
                                        C.c_void_p]),
    "brace_aggregate_host": (C.c_int, [C.c_void_p, C.POINTER(Attack), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "brace_debug_mailbox": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_void_p), C.POINTER(C.c_int64),
                                      C.POINTER(C.c_int32), C.POINTER(C.c_int32)]),
    "brace_set_tuning": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32]),
    "brace_debug_status": (C.c_int, [C.POINTER(C.c_int32)]),
    "brace_minmax_rate_probe": (C.c_int, [C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_int64), C.c_void_p]),
    "brace_aggregate_static": (C.c_int, [C.c_int32, C.c_int64, C.POINTER(Params), C.c_void_p, C.c_int64, C.c_void_p,
                                         C.c_int64, C.c_void_p]),
    "brace_ortho_default_params": (C.c_int, [C.POINTER(OrthoParams)]),
    "brace_ortho_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int32, C.c_int32, C.POINTER(OrthoParams), C.c_int32]),
    "brace_orthogonalize": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.POINTER(OrthoParams), C.c_void_p, C.c_int32,
                                      C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int32, C.c_int64, C.c_int64,
                                      C.c_void_p, C.c_size_t, C.c_void_p]),
    "brace_muon_step": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.POINTER(OrthoParams), C.POINTER(Muon),
                                  C.c_void_p, C.c_size_t, C.c_void_p]),
    "brace_ortho_status": (C.c_int, [C.c_void_p, C.c_void_p]),
    "brace_embedding_lookup": (C.c_int, [C.POINTER(EmbeddingArgs), C.c_void_p]),
    "brace_embedding_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int64, C.c_int64, C.c_int32]),
    "brace_embedding_grad": (C.c_int, [C.POINTER(EmbeddingArgs), C.c_void_p, C.c_size_t, C.c_void_p]),
}

STATIC_SCRATCH_BYTES = 8 * 1024 * 1024


def lib() -> C.CDLL:
    """Load the compiled library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2501_17392_b200.build` "
                               "(there is no CPU fallback)")
        handle = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def status_string(status: int) -> str:
    return lib().brace_status_string(status).decode()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise BraceError(status, where)


def default_params(**over) -> Params:
    p = Params()
    _check(lib().brace_default_params(C.byref(p)), "brace_default_params")
    for k, v in over.items():
        if k == "lambda_":
            k = "lam"
        setattr(p, k, v)
    return p


def workspace_bytes(n: int, d: int, params: Params) -> int:
    return int(lib().brace_workspace_bytes(n, d, C.byref(params)))


# the current stream's handle without a Stream object around it (a microsecond of a call's ten)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def make_attack(kind: int, *, scale=1.0, sigma=1.0, kappa=3.0, prob=0.1, byz_ids=None, noise=None,
                uniform=None, seed=None, round_idx=0) -> Attack:
    """Build the attack descriptor; keeps the id array alive on the returned object.
    With `seed` given the library draws the attack's random numbers itself from
    (seed, round_idx); otherwise `noise` / `uniform` supply them."""
    a = Attack()
    a.kind, a.scale, a.sigma, a.kappa, a.prob = kind, scale, sigma, kappa, prob
    if seed is not None:
        a.draws, a.seed, a.round = DRAWS_GENERATED, int(seed), int(round_idx)
    if byz_ids is not None:
        arr = (C.c_int32 * len(byz_ids))(*[int(i) for i in byz_ids])
        a._ids_keepalive = arr
        a.h_byz_ids = C.cast(arr, C.POINTER(C.c_int32))
    if noise is not None:
        a._noise_keepalive = noise
        a.noise, a.noise_ld = _ptr(noise), noise.stride(0)
    if uniform is not None:
        a._uniform_keepalive = uniform
        a.uniform, a.uniform_ld = _ptr(uniform), uniform.stride(0)
    return a


def draw_matrix_status(what: int, seed: int, round_idx: int, first_client: int, out: torch.Tensor, d: int,
                       mu=0.0, sigma=1.0, stream=None) -> int:
    return lib().brace_draw_matrix(what, seed, round_idx, first_client, out.shape[0], d, _ptr(out), out.stride(0),
                                   float(mu), float(sigma), _stream(stream))


def draw_matrix(what: int, seed: int, round_idx: int, first_client: int, out: torch.Tensor, d: int, mu=0.0,
                sigma=1.0, stream=None):
    """Fill `out` [rows, ld] with the library's own uniform / normal draws of clients
    first_client .. first_client + rows - 1 (the draws attacks 2 and 5 consume)."""
    _check(draw_matrix_status(what, seed, round_idx, first_client, out, d, mu, sigma, stream), "brace_draw_matrix")


def minmax_rate_probe(blocks: int, iters: int, out: torch.Tensor, stream=None) -> int:
    """Launch the min/max calibration kernel; returns the number of operations it performs."""
    ops = C.c_int64(0)
    _check(lib().brace_minmax_rate_probe(blocks, iters, _ptr(out), C.byref(ops), _stream(stream)),
           "brace_minmax_rate_probe")
    return ops.value


def debug_status():
    """(status, code): code of the first index check that failed in a debug build since the last call."""
    code = C.c_int32(0)
    status = lib().brace_debug_status(C.byref(code))
    return status, code.value


def aggregate_static_status(n: int, d: int, params: Params, updates: torch.Tensor, out: torch.Tensor,
                            stream=None) -> int:
    """brace_aggregate_static: a fused round whose mailboxes live in the library's
    built-in scratch array, for callers that cannot allocate a workspace."""
    return lib().brace_aggregate_static(n, d, C.byref(params), _ptr(updates), updates.stride(0), _ptr(out),
                                        out.stride(0), _stream(stream))


def aggregate_static(n: int, d: int, params: Params, updates: torch.Tensor, out: torch.Tensor, stream=None):
    _check(aggregate_static_status(n, d, params, updates, out, stream), "brace_aggregate_static")


class Brace:
    """One aggregation context: n clients, f Byzantine, d coordinates."""

    def __init__(self, n: int, f: int, d: int, params: Params | None = None, device="cuda", host_only=False,
                 workspace: torch.Tensor | None = None):
        self.n, self.f, self.d = n, f, d
        self.params = params if params is not None else default_params()
        self._ctx = C.c_void_p()
        self.workspace = None
        if host_only:
            ws_ptr, ws_bytes = None, 0
        elif workspace is not None:          # caller-owned uint8 device tensor
            self.workspace = workspace
            ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel()
        else:
            need = workspace_bytes(n, d, self.params)
            if need == 0:
                # let brace_init report the precise reason
                need = 256
            self.workspace = torch.empty(need, dtype=torch.uint8, device=device)
            ws_ptr, ws_bytes = self.workspace.data_ptr(), need
        _check(lib().brace_init(C.byref(self._ctx), n, f, d, C.byref(self.params), ws_ptr, ws_bytes, None),
               "brace_init")

    # ---- lifetime
    def close(self):
        if self._ctx:
            lib().brace_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- host queries
    def segment(self, j: int):
        b, e = C.c_int64(), C.c_int64()
        _check(lib().brace_segment(self._ctx, j, C.byref(b), C.byref(e)), "brace_segment")
        return b.value, e.value

    def comm_cost(self, m_bits: int) -> Cost:
        cost = Cost()
        _check(lib().brace_comm_cost(self._ctx, m_bits, C.byref(cost)), "brace_comm_cost")
        return cost

    def last_cuda_error(self) -> int:
        return int(lib().brace_last_cuda_error(self._ctx))

    def set_tuning(self, fused_variant=0, fused_grid=0):
        _check(lib().brace_set_tuning(self._ctx, fused_variant, fused_grid), "brace_set_tuning")

    @property
    def out_words(self) -> int:
        return (self.d + 31) // 32

    def new_output(self, out_ld: int | None = None, device="cuda") -> torch.Tensor:
        if self.params.rule == RULE_SUM:
            ld = out_ld or (self.d + 3) // 4 * 4
            return torch.zeros((self.n, ld), dtype=torch.float32, device=device)
        ld = out_ld or (self.out_words + 3) // 4 * 4
        return torch.zeros((self.n, ld), dtype=torch.int32, device=device)

    # ---- device calls (raw status variants end in _status)
    def inject_attack(self, attack: Attack, honest: torch.Tensor, updates: torch.Tensor, stream=None):
        _check(lib().brace_inject_attack(self._ctx, C.byref(attack), _ptr(honest), honest.stride(0), _ptr(updates),
                                         updates.stride(0), _stream(stream)), "brace_inject_attack")

    def quantize(self, updates: torch.Tensor, q: torch.Tensor, stream=None):
        _check(lib().brace_quantize(self._ctx, _ptr(updates), updates.stride(0), _ptr(q), q.stride(0),
                                    _stream(stream)), "brace_quantize")

    def reduce_scatter_step_status(self, step: int, updates: torch.Tensor, stream=None) -> int:
        return lib().brace_ring_reduce_scatter_step(self._ctx, step, _ptr(updates), updates.stride(0),
                                                    _stream(stream))

    def reduce_scatter_step(self, step: int, updates: torch.Tensor, stream=None):
        _check(self.reduce_scatter_step_status(step, updates, stream), "brace_ring_reduce_scatter_step")

    def consensus_status(self, out: torch.Tensor, stream=None) -> int:
        return lib().brace_consensus(self._ctx, _ptr(out), out.stride(0), _stream(stream))

    def consensus(self, out: torch.Tensor, stream=None):
        _check(self.consensus_status(out, stream), "brace_consensus")

    def allgather_step_status(self, step: int, out: torch.Tensor, stream=None) -> int:
        return lib().brace_ring_allgather_step(self._ctx, step, _ptr(out), out.stride(0), _stream(stream))

    def allgather_step(self, step: int, out: torch.Tensor, stream=None):
        _check(self.allgather_step_status(step, out, stream), "brace_ring_allgather_step")

    def aggregate_status(self, updates: torch.Tensor, out: torch.Tensor, stream=None) -> int:
        return lib().brace_aggregate(self._ctx, _ptr(updates), updates.stride(0), _ptr(out), out.stride(0),
                                     _stream(stream))

    def aggregate(self, updates: torch.Tensor, out: torch.Tensor, stream=None):
        _check(self.aggregate_status(updates, out, stream), "brace_aggregate")

    def apply_update_status(self, out: torch.Tensor, weights: torch.Tensor, eta: float, stream=None) -> int:
        return lib().brace_apply_update(self._ctx, _ptr(out), out.stride(0), _ptr(weights), weights.stride(0),
                                        float(eta), _stream(stream))

    def apply_update(self, out: torch.Tensor, weights: torch.Tensor, eta: float, stream=None):
        """Each client's parameter row moves by the aggregate in its output row."""
        _check(self.apply_update_status(out, weights, eta, stream), "brace_apply_update")

    def coordinate_stat_status(self, kind: int, trim: int, updates: torch.Tensor, result: torch.Tensor,
                               stream=None) -> int:
        return lib().brace_coordinate_stat(self._ctx, kind, trim, _ptr(updates), updates.stride(0), _ptr(result),
                                           _stream(stream))

    def coordinate_stat(self, kind: int, trim: int, updates: torch.Tensor, result: torch.Tensor, stream=None):
        """Coordinate-wise median / trimmed mean of the n rows into one float32 vector."""
        _check(self.coordinate_stat_status(kind, trim, updates, result, stream), "brace_coordinate_stat")

    def aggregate_host(self, attack: Attack | None, h_updates: torch.Tensor, h_out: torch.Tensor,
                       d_updates: torch.Tensor, d_out: torch.Tensor, d_noise=None, d_uniform=None, stream=None):
        """Host-buffer round: h_updates / h_out (and attack.noise / uniform) are CPU
        tensors, ideally pinned; the d_* tensors are device staging of the same shapes."""
        assert h_updates.stride(0) == d_updates.stride(0) and h_out.stride(0) == d_out.stride(0)
        _check(lib().brace_aggregate_host(self._ctx, C.byref(attack) if attack is not None else None,
                                          _ptr(h_updates), h_updates.stride(0), _ptr(h_out), h_out.stride(0),
                                          _ptr(d_updates), _ptr(d_noise), _ptr(d_uniform), _ptr(d_out),
                                          _stream(stream)), "brace_aggregate_host")

    def debug_mailbox(self, client: int, hops_back: int = 0):
        """(device pointer, length, sub-vector id, entry bytes) of a client's mailbox."""
        p, ln, seg, eb = C.c_void_p(), C.c_int64(), C.c_int32(), C.c_int32()
        _check(lib().brace_debug_mailbox(self._ctx, client, hops_back, C.byref(p), C.byref(ln), C.byref(seg),
                                         C.byref(eb)), "brace_debug_mailbox")
        return p.value, ln.value, seg.value, eb.value

    def mailbox_tensor(self, client: int, hops_back: int = 0) -> tuple[int, torch.Tensor]:
        """(sub-vector id, copy of the mailbox contents as a CPU int64/float32 tensor)."""
        p, ln, seg, eb = self.debug_mailbox(client, hops_back)
        off = p - self.workspace.data_ptr()
        raw = self.workspace[off: off + ln * eb]
        dt = {1: torch.int8, 2: torch.int16, 4: torch.float32}[eb]
        return seg, raw.view(dt).cpu()


# ---- operators of a language model's round -----------------------------------------------------------------------

_FLOATS = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}
_ID_BYTES = {torch.int64: 8, torch.int32: 4}
_EMBEDDING = struct.Struct("@ii10q4if")       # the fields of EmbeddingArgs


def _launch_stream(stream, device: int, same: bool) -> int:
    """The stream of a call whose tensors are on `device` (all of them: `same`).  A kernel that is handed another device's
    memory, or the host's, would fault."""
    if not same or device < 0:
        raise ValueError("the tensors and the workspace have to be on one GPU")
    if device != torch.cuda.current_device():
        raise ValueError(f"the tensors are on GPU {device}, the current one is {torch.cuda.current_device()}")
    if stream is None and _raw_stream is not None:
        return _raw_stream(device)
    return _stream(stream)


def ortho_params(**over) -> OrthoParams:
    p = OrthoParams()
    _check(lib().brace_ortho_default_params(C.byref(p)), "brace_ortho_default_params")
    for k, v in over.items():
        setattr(p, k, v)
    return p


def ortho_workspace_bytes(batch: int, rows: int, cols: int, params: OrthoParams, out_type: int = TYPE_F32) -> int:
    return int(lib().brace_ortho_workspace_bytes(batch, rows, cols, C.byref(params), out_type))


class Orthogonalizer:
    """Workspace and parameters of the orthogonalised update of `batch` matrices of rows x cols.

    Matrices are float32, bfloat16 or float16 tensors [batch, rows, cols] (or [rows, cols] where batch is 1) whose
    last stride is 1; an int32 tensor is a row of packed bits as a round leaves it, with the matrices one after the
    other from `bit_offset` on.  All are on the current GPU.  An object serves one host thread, and one stream at a time (its
    workspace)."""

    def __init__(self, rows: int, cols: int, batch: int = 1, params: OrthoParams | None = None, device="cuda",
                 workspace: torch.Tensor | None = None):
        self.batch, self.rows, self.cols = batch, rows, cols
        self.params = params if params is not None else ortho_params()
        if workspace is None:
            need = ortho_workspace_bytes(batch, rows, cols, self.params)
            # 0: the arguments are refused; the calls give the reason
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
        self.workspace = workspace
        self._step = Muon()
        self._computed = False      # whether a call has written the workspace's status

    def _matrix(self, t: torch.Tensor, name: str):
        """(element type, ld, stride between matrices) of a tensor argument."""
        shape = t.shape
        if shape != (self.batch, self.rows, self.cols) and not (self.batch == 1 and shape == (self.rows, self.cols)):
            raise ValueError(f"{name} has shape {tuple(shape)}, not {(self.batch, self.rows, self.cols)}")
        kind = _FLOATS.get(t.dtype)
        if kind is None:
            raise ValueError(f"{name} is of type {t.dtype}")
        st = t.stride()
        if self.cols > 1 and st[-1] != 1:
            raise ValueError(f"{name}: the last dimension is not contiguous")
        # the stride of a dimension of one (or no) element has no meaning
        return kind, st[-2] if self.rows > 1 else max(self.cols, 1), st[0] if self.batch > 1 else 0

    def _update(self, g: torch.Tensor, name: str, bit_offset: int):
        if g.dtype == torch.int32:
            need = bit_offset + self.batch * self.rows * self.cols
            if g.dim() != 1 or (g.numel() > 1 and g.stride(0) != 1) or bit_offset < 0 or 32 * g.numel() < need:
                raise ValueError(f"{name}: packed bits are a contiguous row of at least {need} bits")
            return TYPE_BITS, self.cols, self.rows * self.cols
        return self._matrix(g, name)

    def orthogonalize_status(self, g: torch.Tensor, out: torch.Tensor, bit_offset: int = 0, stream=None) -> int:
        gt, gld, gs = self._update(g, "g", bit_offset)
        ot, old, os_ = self._matrix(out, "out")
        at = g.get_device()
        st = _launch_stream(stream, at, at == out.get_device() == self.workspace.get_device())
        status = lib().brace_orthogonalize(self.batch, self.rows, self.cols, self.params, g.data_ptr(), gt, gld, gs,
                                           bit_offset, out.data_ptr(), ot, old, os_, self.workspace.data_ptr(),
                                           self.workspace.numel(), st)
        self._computed |= status == OK and out.numel() > 0
        return status

    def orthogonalize(self, g: torch.Tensor, out: torch.Tensor, bit_offset: int = 0, stream=None):
        """out = g with its singular values pushed to 1."""
        _check(self.orthogonalize_status(g, out, bit_offset, stream), "brace_orthogonalize")

    def muon_step_status(self, grad: torch.Tensor, momentum: torch.Tensor, weights: torch.Tensor, lr: float,
                         beta: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, scale: float = 1.0,
                         bit_offset: int = 0, momentum_out: torch.Tensor | None = None,
                         weights_out: torch.Tensor | None = None, stream=None) -> int:
        momentum_out = momentum if momentum_out is None else momentum_out
        weights_out = weights if weights_out is None else weights_out
        s = self._step
        s.grad_type, s.ld_grad, s.stride_grad = self._update(grad, "grad", bit_offset)
        s.d_grad, s.bit_offset = grad.data_ptr(), bit_offset
        for t, name in ((momentum, "momentum"), (momentum_out, "momentum_out")):
            if t.dtype != torch.float32:
                raise ValueError(f"{name} is of type {t.dtype}, not float32")
        _, s.ld_momentum, s.stride_momentum = self._matrix(momentum, "momentum")
        _, s.ld_momentum_out, s.stride_momentum_out = self._matrix(momentum_out, "momentum_out")
        s.d_momentum, s.d_momentum_out = momentum.data_ptr(), momentum_out.data_ptr()
        replicas = 1
        s.replica_weights = s.replica_weights_out = 0
        w, wo = weights, weights_out
        if weights.dim() == 4:      # [replicas, batch, rows, cols]
            replicas = weights.shape[0]
            if weights_out.dim() != 4 or weights_out.shape[0] != replicas or replicas < 1:
                raise ValueError("weights and weights_out have different shapes")
            s.replica_weights, s.replica_weights_out = weights.stride(0), weights_out.stride(0)
            w, wo = weights[0], weights_out[0]
        if w.dtype != wo.dtype:
            raise ValueError("weights and weights_out have different types")
        s.weights_type, s.ld_weights, s.stride_weights = self._matrix(w, "weights")
        _, s.ld_weights_out, s.stride_weights_out = self._matrix(wo, "weights_out")
        s.d_weights, s.d_weights_out, s.replicas = w.data_ptr(), wo.data_ptr(), replicas
        s.nesterov, s.beta, s.lr, s.weight_decay, s.scale = int(nesterov), beta, lr, weight_decay, scale
        at = grad.get_device()
        st = _launch_stream(stream, at, at == momentum.get_device() == momentum_out.get_device() == weights.get_device()
                            == weights_out.get_device() == self.workspace.get_device())
        status = lib().brace_muon_step(self.batch, self.rows, self.cols, self.params, s, self.workspace.data_ptr(),
                                       self.workspace.numel(), st)
        self._computed |= status == OK and momentum.numel() > 0
        return status

    def muon_step(self, grad: torch.Tensor, momentum: torch.Tensor, weights: torch.Tensor, lr: float,
                  beta: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, scale: float = 1.0,
                  bit_offset: int = 0, momentum_out: torch.Tensor | None = None,
                  weights_out: torch.Tensor | None = None, stream=None):
        """One step of momentum, orthogonalisation and weight update, in place unless *_out are given.  Weights of
        shape [replicas, batch, rows, cols] all take the same step."""
        _check(self.muon_step_status(grad, momentum, weights, lr, beta, nesterov, weight_decay, scale, bit_offset,
                                     momentum_out, weights_out, stream), "brace_muon_step")

    def check(self, stream=None):
        """Wait for the stream; raise if a bounded device-side wait of the last call ran out."""
        if not self._computed:      # there was none: the workspace holds whatever it held
            (torch.cuda.current_stream() if stream is None else stream).synchronize()
            return
        _check(lib().brace_ortho_status(self.workspace.data_ptr(), _stream(stream)), "brace_ortho_status")


class Embedding:
    """The embedding table of `clients` clients with up to `tokens` ids each per call.

    Tables (and their gradients) are tensors [clients, vocab, dim] -- views of the clients' rows of weights or updates
    -- or [vocab, dim]; activations [clients, n, dim] or [n, dim]; ids int64 or int32 [clients, n] or [n].  The last
    stride is 1.  All are on the current GPU.  `grad` = False leaves the gradient's workspace out.  An object serves one
    host thread, and one stream at a time (its workspace)."""

    def __init__(self, vocab: int, dim: int, tokens: int, clients: int = 1, grad: bool = True, device="cuda",
                 workspace: torch.Tensor | None = None):
        self.clients, self.vocab, self.dim, self.tokens = clients, vocab, dim, tokens
        if grad and workspace is None:
            need = int(lib().brace_embedding_workspace_bytes(clients, tokens, vocab, dim))
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
        self.workspace = workspace
        self._args = EmbeddingArgs()

    def _fill(self, table: torch.Tensor, ids: torch.Tensor, act: torch.Tensor, scale: float, shared: bool,
              accumulate: bool = False):
        c, d, e = self.clients, self.dim, self._args
        shape = ids.shape
        n = shape[-1] if len(shape) else 0
        if (shape != (c, n) and (c != 1 or shape != (n,))) or n > self.tokens:
            raise ValueError(f"ids have shape {tuple(shape)}, not {(c, n)} with at most {self.tokens} tokens")
        id_bytes, id_stride = _ID_BYTES.get(ids.dtype), ids.stride()
        if id_bytes is None or (n > 1 and id_stride[-1] != 1):
            raise ValueError("ids are int64 or int32 with a contiguous last dimension")
        if table.shape != (c, self.vocab, d) and not ((c == 1 or shared) and table.shape == (self.vocab, d)):
            raise ValueError(f"table has shape {tuple(table.shape)}, not {(c, self.vocab, d)}")
        if act.shape != (c, n, d) and not (c == 1 and act.shape == (n, d)):
            raise ValueError(f"activations have shape {tuple(act.shape)}, not {(c, n, d)}")
        table_type, act_type = _FLOATS.get(table.dtype), _FLOATS.get(act.dtype)
        if table_type is None or act_type is None:
            raise ValueError(f"table and activations are of type {table.dtype} and {act.dtype}")
        ts, as_ = table.stride(), act.stride()
        if d > 1 and (ts[-1] != 1 or as_[-1] != 1):
            raise ValueError("the last dimension of table and activations is contiguous")
        # the stride of a dimension of one element has no meaning
        _EMBEDDING.pack_into(e, 0, c, d, n, self.vocab, table.data_ptr(), ts[-2] if self.vocab > 1 else d,
                             ts[0] if c > 1 and len(ts) == 3 else 0, ids.data_ptr(), id_stride[0] if c > 1 else 0,
                             act.data_ptr(), as_[-2] if n > 1 else d, as_[0] if c > 1 else 0, table_type, act_type,
                             id_bytes, accumulate, scale)
        return e

    def lookup_status(self, table, ids, out, scale: float = 1.0, stream=None) -> int:
        e, at = self._fill(table, ids, out, scale, True), table.get_device()
        return lib().brace_embedding_lookup(e, _launch_stream(stream, at, at == ids.get_device() == out.get_device()))

    def lookup(self, table: torch.Tensor, ids: torch.Tensor, out: torch.Tensor, scale: float = 1.0, stream=None):
        """out[c, t] = scale * table[c, ids[c, t]]; 0 for an id outside the table.  A two-dimensional table serves
        all clients."""
        _check(self.lookup_status(table, ids, out, scale, stream), "brace_embedding_lookup")

    def grad_status(self, dy, ids, grad, scale: float = 1.0, accumulate: bool = False, stream=None) -> int:
        e, ws = self._fill(grad, ids, dy, scale, False, accumulate), self.workspace
        if ws is None:      # refused
            return lib().brace_embedding_grad(e, 0, 0, 0)
        at = grad.get_device()
        st = _launch_stream(stream, at, at == ids.get_device() == dy.get_device() == ws.get_device())
        return lib().brace_embedding_grad(e, ws.data_ptr(), ws.numel(), st)

    def grad(self, dy: torch.Tensor, ids: torch.Tensor, grad: torch.Tensor, scale: float = 1.0,
             accumulate: bool = False, stream=None):
        """grad[c, v] = scale * the sum of dy[c, t] over the tokens with id v (added to grad with `accumulate`)."""
        _check(self.grad_status(dy, ids, grad, scale, accumulate, stream), "brace_embedding_grad")
