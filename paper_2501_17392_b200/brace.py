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
CLIP_PROPAGATE, CLIP_ZERO = 0, 1


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


class LayerNormArgs(C.Structure):
    _fields_ = [("clients", C.c_int32), ("dim", C.c_int32), ("rows", C.c_int64), ("d_x", C.c_void_p),
                ("ld_x", C.c_int64), ("stride_x", C.c_int64), ("d_weight", C.c_void_p), ("stride_weight", C.c_int64),
                ("d_bias", C.c_void_p), ("stride_bias", C.c_int64), ("d_y", C.c_void_p), ("ld_y", C.c_int64),
                ("stride_y", C.c_int64), ("d_mean", C.c_void_p), ("d_rstd", C.c_void_p), ("stride_stats", C.c_int64),
                ("d_dx", C.c_void_p), ("ld_dx", C.c_int64), ("stride_dx", C.c_int64), ("d_dweight", C.c_void_p),
                ("stride_dweight", C.c_int64), ("d_dbias", C.c_void_p), ("stride_dbias", C.c_int64),
                ("x_type", C.c_int32), ("y_type", C.c_int32), ("weight_type", C.c_int32), ("grad_type", C.c_int32),
                ("accumulate", C.c_int32), ("eps", C.c_float)]


class TensorArgs(C.Structure):
    _fields_ = [("d_in", C.c_void_p), ("d_out", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64),
                ("ld_in", C.c_int64), ("stride_in", C.c_int64), ("ld_out", C.c_int64), ("stride_out", C.c_int64),
                ("in_type", C.c_int32), ("out_type", C.c_int32)]


class Heads(C.Structure):
    _fields_ = [("d", C.c_void_p), ("ld", C.c_int64), ("head", C.c_int64), ("stride", C.c_int64)]


class WindowAttentionArgs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("tokens", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("dim", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32), ("type", C.c_int32),
                ("scale", C.c_float), ("d_lengths", C.c_void_p), ("q", Heads), ("k", Heads), ("v", Heads),
                ("out", Heads), ("d_lse", C.c_void_p), ("head_lse", C.c_int64), ("stride_lse", C.c_int64),
                ("dout", Heads), ("dq", Heads), ("dk", Heads), ("dv", Heads)]


# where the tensors lie in it
_Q, _K, _V, _OUT, _DOUT, _DQ, _DK, _DV = (getattr(WindowAttentionArgs, f).offset
                                          for f in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"))


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
    "brace_layer_norm_forward": (C.c_int, [C.POINTER(LayerNormArgs), C.c_void_p]),
    "brace_layer_norm_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int64, C.c_int32]),
    "brace_layer_norm_grad": (C.c_int, [C.POINTER(LayerNormArgs), C.c_void_p, C.c_size_t, C.c_void_p]),
    "brace_window_attention_forward": (C.c_int, [C.POINTER(WindowAttentionArgs), C.c_void_p]),
    "brace_window_attention_workspace_bytes": (C.c_size_t, [C.c_int32] * 6),
    "brace_window_attention_window_workspace_bytes": (C.c_size_t, [C.c_int32] * 7),
    "brace_window_attention_grad": (C.c_int, [C.POINTER(WindowAttentionArgs), C.c_void_p, C.c_size_t, C.c_void_p]),
    "brace_clip_workspace_bytes": (C.c_size_t, [C.c_int32, C.POINTER(TensorArgs), C.c_int32]),
    "brace_gradient_norm": (C.c_int, [C.c_int32, C.POINTER(TensorArgs), C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t,
                                      C.c_void_p]),
    "brace_gradient_clip": (C.c_int, [C.c_int32, C.POINTER(TensorArgs), C.c_int32, C.c_float, C.c_float, C.c_int32,
                                      C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
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
_LAYER_NORM = struct.Struct("@ii21q5if")      # of LayerNormArgs
_ATTENTION = struct.Struct("@8ifq")           # of WindowAttentionArgs, up to the tensors
_HEADS = struct.Struct("@4q")                 # of Heads


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


class LayerNorm:
    """Layer norm of the activations of `clients` clients with up to `rows` rows each per call.

    Activations are tensors [clients, n, dim] or [n, dim], weight and bias [clients, dim] -- pieces of the clients' rows of
    weights -- or [dim] (forward: one for all clients), their gradients [clients, dim] or, of one client, [dim]; mean and
    rstd float32 [clients, n] or [n].  The last stride is 1.  All are on the current GPU.  `grad` = False leaves the
    gradient's workspace out.  An object serves one host thread, and one stream at a time (its workspace)."""

    def __init__(self, dim: int, rows: int, clients: int = 1, eps: float = 1e-5, grad: bool = True, device="cuda",
                 workspace: torch.Tensor | None = None):
        self.dim, self.rows, self.clients, self.eps = dim, rows, clients, eps
        if grad and workspace is None:
            need = int(lib().brace_layer_norm_workspace_bytes(clients, rows, dim))
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
        self.workspace = workspace
        self._args = LayerNormArgs()

    def _rows(self, t: torch.Tensor, name: str, n: int):
        """(element type, ld, stride between clients) of activations."""
        c, d, shape = self.clients, self.dim, t.shape
        if shape != (c, n, d) and not (c == 1 and shape == (n, d)):
            raise ValueError(f"{name} has shape {tuple(shape)}, not {(c, n, d)}")
        kind, st = _FLOATS.get(t.dtype), t.stride()
        if kind is None or (st[-1] != 1 and d > 1):
            raise ValueError(f"{name} is of type {t.dtype} with strides {st}")
        # the stride of a dimension of one element has no meaning
        return kind, st[-2] if n > 1 else d, st[0] if c > 1 else 0

    def _vector(self, t: torch.Tensor, name: str, shared: bool):
        """(element type, stride between clients) of a weight, a bias or a gradient of them."""
        c, d, shape = self.clients, self.dim, t.shape
        if shape != (c, d) and not ((c == 1 or shared) and shape == (d,)):
            raise ValueError(f"{name} has shape {tuple(shape)}, not {(c, d)}")
        kind, st = _FLOATS.get(t.dtype), t.stride()
        if kind is None or (st[-1] != 1 and d > 1):
            raise ValueError(f"{name} is of type {t.dtype} with strides {st}")
        return kind, st[0] if c > 1 and len(st) == 2 else 0

    def _pair(self, t, u, name: str, shared: bool):
        """(pointer, stride) of a weight and a bias, or of their gradients, and their element type."""
        tp = ts = up = us = 0
        kind = other = None
        if t is not None:
            kind, ts = self._vector(t, name + "weight", shared)
            tp = t.data_ptr()
        if u is not None:
            other, us = self._vector(u, name + "bias", shared)
            up = u.data_ptr()
            if kind is not None and kind != other:
                raise ValueError(f"{name}weight and {name}bias have different types")
        return tp, ts, up, us, kind if kind is not None else other if other is not None else TYPE_F32

    def _stat(self, t: torch.Tensor, name: str, n: int) -> int:
        """Stride between the clients of a row's mean or rstd."""
        c, shape, st = self.clients, t.shape, t.stride()
        if t.dtype is not torch.float32 or (shape != (c, n) and not (c == 1 and shape == (n,))):
            raise ValueError(f"{name} has shape {tuple(shape)} and type {t.dtype}, not {(c, n)} and float32")
        if st[-1] != 1 and n > 1:
            raise ValueError(f"{name}: the last dimension is not contiguous")
        return st[0] if c > 1 else n

    def _count(self, x: torch.Tensor) -> int:
        n = x.shape[-2] if x.dim() >= 2 else -1
        if not 0 <= n <= self.rows:
            raise ValueError(f"x has shape {tuple(x.shape)}: at most {self.rows} rows")
        return n

    def _stats(self, mean, rstd, n: int) -> int:
        m, r = None if mean is None else self._stat(mean, "mean", n), None if rstd is None else self._stat(rstd, "rstd", n)
        if m is not None and r is not None and m != r:
            raise ValueError("mean and rstd have different strides")
        return m if m is not None else r if r is not None else n

    def forward_status(self, x, y, weight=None, bias=None, mean=None, rstd=None, stream=None) -> int:
        n, at = self._count(x), x.get_device()
        xt, xl, xs = self._rows(x, "x", n)
        yt, yl, ys = self._rows(y, "y", n)
        wp, ws, bp, bs, wt = self._pair(weight, bias, "", True)
        same = y.get_device() == at
        for t in (weight, bias, mean, rstd):
            same = same and (t is None or t.get_device() == at)
        e = self._args
        _LAYER_NORM.pack_into(e, 0, self.clients, self.dim, n, x.data_ptr(), xl, xs, wp, ws, bp, bs, y.data_ptr(), yl, ys,
                              _ptr(mean), _ptr(rstd), self._stats(mean, rstd, n), 0, 0, 0, 0, 0, 0, 0, xt, yt, wt, TYPE_F32, 0,
                              self.eps)
        return lib().brace_layer_norm_forward(e, _launch_stream(stream, at, same))

    def forward(self, x: torch.Tensor, y: torch.Tensor, weight: torch.Tensor | None = None,
                bias: torch.Tensor | None = None, mean: torch.Tensor | None = None, rstd: torch.Tensor | None = None,
                stream=None):
        """y = (x - mean) rstd weight + bias; mean and rstd of the rows are written where they are given."""
        _check(self.forward_status(x, y, weight, bias, mean, rstd, stream), "brace_layer_norm_forward")

    def grad_status(self, dy, x, mean, rstd, dx, weight=None, dweight=None, dbias=None, accumulate: bool = False,
                    stream=None) -> int:
        n, at, buf = self._count(x), x.get_device(), self.workspace
        xt, xl, xs = self._rows(x, "x", n)
        yt, yl, ys = self._rows(dy, "dy", n)
        kind, dl, ds = self._rows(dx, "dx", n)
        if kind != xt:
            raise ValueError(f"dx is of type {dx.dtype}, x of {x.dtype}")
        wp, ws, _, _, wt = self._pair(weight, None, "", True)
        gp, gs, hp, hs, gt = self._pair(dweight, dbias, "d", False)
        same = dy.get_device() == at == dx.get_device() == mean.get_device() == rstd.get_device()
        for t in (weight, dweight, dbias, buf):
            same = same and (t is None or t.get_device() == at)
        e = self._args
        _LAYER_NORM.pack_into(e, 0, self.clients, self.dim, n, x.data_ptr(), xl, xs, wp, ws, 0, 0, dy.data_ptr(), yl, ys,
                              mean.data_ptr(), rstd.data_ptr(), self._stats(mean, rstd, n), dx.data_ptr(), dl, ds, gp, gs, hp, hs,
                              xt, yt, wt, gt, accumulate, self.eps)
        if buf is None:      # refused
            return lib().brace_layer_norm_grad(e, 0, 0, 0)
        return lib().brace_layer_norm_grad(e, buf.data_ptr(), buf.numel(), _launch_stream(stream, at, same))

    def grad(self, dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, dx: torch.Tensor,
             weight: torch.Tensor | None = None, dweight: torch.Tensor | None = None,
             dbias: torch.Tensor | None = None, accumulate: bool = False, stream=None):
        """dx, and (where they are given) the gradients of weight and bias, added to what these hold with `accumulate`."""
        _check(self.grad_status(dy, x, mean, rstd, dx, weight, dweight, dbias, accumulate, stream),
               "brace_layer_norm_grad")


class WindowAttention:
    """Causal attention over `batch` sequences of up to `tokens` tokens each, with a sliding window and `sinks` first
    tokens that stay visible: query i sees key j iff j <= i and (i - j < window or j < sinks).

    Queries, outputs and their gradients are tensors [batch, n, heads, dim], keys and values [batch, n, kv_heads, dim], all
    of one type (float32, bfloat16 or float16) with a contiguous last dimension -- views of one projection's result, for
    instance; lse is float32 [batch, heads, n], lengths int32 [batch]: the tokens of each sequence, rows behind them are 0
    in every result.  All are on the current GPU.  `scale` is 1 / sqrt(dim) where it is not given.  `grad` = False leaves
    the gradient's workspace out.  An object serves one host thread, and one stream at a time (its workspace)."""

    def __init__(self, heads: int, dim: int, tokens: int, batch: int = 1, kv_heads: int | None = None, window: int = 1024,
                 sinks: int = 0, scale: float | None = None, grad: bool = True, device="cuda",
                 workspace: torch.Tensor | None = None):
        self.heads, self.dim, self.tokens, self.batch = heads, dim, tokens, batch
        self.kv_heads = heads if kv_heads is None else kv_heads
        self.window, self.sinks, self.scale = window, sinks, dim ** -0.5 if scale is None else scale
        if grad and workspace is None:
            need = int(lib().brace_window_attention_window_workspace_bytes(batch, tokens, heads, self.kv_heads, dim, window, sinks))
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
        self.workspace = workspace
        self._args = WindowAttentionArgs()

    def _heads(self, field: int, t: torch.Tensor, name: str, n: int, heads: int, dtype):
        b, d, shape, st = self.batch, self.dim, t.shape, t.stride()
        if shape != (b, n, heads, d):
            raise ValueError(f"{name} has shape {tuple(shape)}, not {(b, n, heads, d)}")
        if t.dtype is not dtype or (st[3] != 1 and d > 1):
            raise ValueError(f"{name} is of type {t.dtype} with strides {st}, q of type {dtype}")
        # the stride of a dimension of one element has no meaning
        _HEADS.pack_into(self._args, field, t.data_ptr(), st[1], st[2] if heads > 1 else 0, st[0] if b > 1 else 0)

    def _fill(self, q, k, v, out, lse, lengths) -> WindowAttentionArgs:
        e, n, dtype = self._args, q.shape[1] if q.dim() == 4 else -1, q.dtype
        kind, h, g = _FLOATS.get(dtype), self.heads, self.kv_heads
        if not 0 <= n <= self.tokens or kind is None:
            raise ValueError(f"q has shape {tuple(q.shape)} and type {dtype}: at most {self.tokens} tokens")
        self._heads(_Q, q, "q", n, h, dtype)
        self._heads(_K, k, "k", n, g, dtype)
        self._heads(_V, v, "v", n, g, dtype)
        self._heads(_OUT, out, "out", n, h, dtype)
        if lse is not None:
            st = lse.stride()
            if lse.dtype is not torch.float32 or lse.shape != (self.batch, h, n) or (st[2] != 1 and n > 1):
                raise ValueError(f"lse has shape {tuple(lse.shape)} and type {lse.dtype}, not {(self.batch, h, n)} and float32")
            e.stride_lse, e.head_lse = st[0], st[1]
        if lengths is not None and (lengths.dtype is not torch.int32 or lengths.shape != (self.batch,)
                                    or (self.batch > 1 and lengths.stride(0) != 1)):
            raise ValueError(f"lengths have shape {tuple(lengths.shape)} and type {lengths.dtype}, not {(self.batch,)} and int32")
        _ATTENTION.pack_into(e, 0, self.batch, n, h, g, self.dim, self.window, self.sinks, kind, self.scale, _ptr(lengths))
        e.d_lse = _ptr(lse)
        return e

    def forward_status(self, q, k, v, out, lse=None, lengths=None, stream=None) -> int:
        e, at = self._fill(q, k, v, out, lse, lengths), q.get_device()
        same = (k.get_device() == at == v.get_device() == out.get_device() and (lse is None or lse.get_device() == at)
                and (lengths is None or lengths.get_device() == at))
        return lib().brace_window_attention_forward(e, _launch_stream(stream, at, same))

    def forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                lse: torch.Tensor | None = None, lengths: torch.Tensor | None = None, stream=None):
        """out = softmax(scale q k^T over the keys seen) v; the logarithms of the softmax's sums where lse is given."""
        _check(self.forward_status(q, k, v, out, lse, lengths, stream), "brace_window_attention_forward")

    def grad_status(self, dout, q, k, v, out, lse, dq, dk, dv, lengths=None, stream=None) -> int:
        e, ws, n = self._fill(q, k, v, out, lse, lengths), self.workspace, q.shape[1]
        self._heads(_DOUT, dout, "dout", n, self.heads, q.dtype)
        self._heads(_DQ, dq, "dq", n, self.heads, q.dtype)
        self._heads(_DK, dk, "dk", n, self.kv_heads, q.dtype)
        self._heads(_DV, dv, "dv", n, self.kv_heads, q.dtype)
        if ws is None:      # refused
            return lib().brace_window_attention_grad(e, 0, 0, 0)
        at = q.get_device()
        same = all(t is None or t.get_device() == at for t in (dout, k, v, out, lse, dq, dk, dv, lengths, ws))
        return lib().brace_window_attention_grad(e, ws.data_ptr(), ws.numel(), _launch_stream(stream, at, same))

    def grad(self, dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
             lse: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor, dv: torch.Tensor,
             lengths: torch.Tensor | None = None, stream=None):
        """dq, dk and dv of sum(out * dout); out and lse are the forward pass's."""
        _check(self.grad_status(dout, q, k, v, out, lse, dq, dk, dv, lengths, stream), "brace_window_attention_grad")


class GradientClip:
    """Every client's gradient norm over a list of tensors, and the tensors clipped by it.

    A tensor is [clients, ...], one client's part of it contiguous or a matrix of contiguous rows, float32, bfloat16 or
    float16; `outs` are tensors of the same shapes (pieces of the update matrix, for instance) that the clipped gradients
    are written to, without them clipping is in place.  All are on the current GPU.  The object is a plan: it keeps the
    tensors, and every call works on what they hold then.  It serves one host thread, and one stream at a time (its
    workspace)."""

    def __init__(self, tensors, outs=None, workspace: torch.Tensor | None = None):
        self.tensors = list(tensors)
        self.outs = self.tensors if outs is None else list(outs)
        if not self.tensors or len(self.outs) != len(self.tensors):
            raise ValueError(f"{len(self.tensors)} tensors and {len(self.outs)} outputs")
        self.clients = self.tensors[0].shape[0] if self.tensors[0].dim() else 0
        self._list = (TensorArgs * len(self.tensors))()
        for e, x, y in zip(self._list, self.tensors, self.outs):
            if x.dim() < 1 or x.shape[0] != self.clients or y.shape != x.shape:
                raise ValueError(f"a tensor has shape {tuple(x.shape)}, its output {tuple(y.shape)}; {self.clients} clients")
            e.in_type, e.out_type = (_FLOATS.get(t.dtype, -1) for t in (x, y))
            if e.in_type < 0 or e.out_type < 0:
                raise ValueError(f"a tensor is of type {x.dtype}, its output of {y.dtype}")
            e.d_in, e.d_out = x.data_ptr(), y.data_ptr()
            e.rows, e.cols, e.ld_in, e.ld_out = self._layout(x, y)
            many = self.clients > 1
            e.stride_in, e.stride_out = (x.stride(0), y.stride(0)) if many else (0, 0)
        self._device = self.tensors[0].get_device()
        self._same = all(t.get_device() == self._device for t in self.tensors + self.outs)
        if workspace is None:
            need = int(lib().brace_clip_workspace_bytes(self.clients, self._list, len(self.tensors)))
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=self.tensors[0].device)
        self.workspace = workspace

    @staticmethod
    def _layout(x, y):
        """(rows, columns, ld of x, ld of y) of one client's part."""
        shape = list(x.shape[1:])
        if x.numel() == 0:
            return 0, 0, 0, 0
        sizes = [(n, s, t) for n, s, t in zip(shape, x.stride()[1:], y.stride()[1:]) if n > 1]
        merged = []          # from the smallest strides on: (size, stride of x, stride of y), runs joined
        for n, s, t in sorted(sizes, key=lambda d: d[1:]):
            if merged and s == merged[-1][0] * merged[-1][1] and t == merged[-1][0] * merged[-1][2]:
                merged[-1] = (n * merged[-1][0], merged[-1][1], merged[-1][2])
            else:
                merged.append((n, s, t))
        if merged and merged[0][1:] != (1, 1):
            merged.insert(0, (1, 1, 1))
        if len(merged) > 2:
            raise ValueError(f"a tensor of shape {tuple(x.shape)} with strides {x.stride()} and {y.stride()} is neither "
                             "contiguous nor a matrix of contiguous rows")
        if len(merged) < 2:
            n = merged[0][0] if merged else 1
            return 1, n, n, n
        return merged[1][0], merged[0][0], merged[1][1], merged[1][2]

    def _norms(self, norms):
        if norms is not None and (norms.dtype != torch.float32 or norms.shape != (self.clients,)
                                  or (self.clients > 1 and norms.stride(0) != 1)):
            raise ValueError(f"norms have shape {tuple(norms.shape)} and type {norms.dtype}, not {(self.clients,)} and float32")
        return _ptr(norms)

    def _stream(self, stream, norms):
        at = self._device
        return _launch_stream(stream, at, self._same and self.workspace.get_device() == at
                              and (norms is None or norms.get_device() == at))

    def norms_status(self, norms: torch.Tensor, stream=None) -> int:
        to, st = self._norms(norms), self._stream(stream, norms)
        return lib().brace_gradient_norm(self.clients, self._list, len(self.tensors), to, self.workspace.data_ptr(),
                                         self.workspace.numel(), st)

    def norms(self, norms: torch.Tensor, stream=None):
        """norms[c] = the 2-norm of all of client c's tensors together."""
        _check(self.norms_status(norms, stream), "brace_gradient_norm")

    def clip_status(self, max_norm: float, norms: torch.Tensor | None = None, eps: float = 1e-6,
                    nonfinite: int = CLIP_PROPAGATE, stream=None) -> int:
        to, st = self._norms(norms), self._stream(stream, norms)
        return lib().brace_gradient_clip(self.clients, self._list, len(self.tensors), max_norm, eps, nonfinite, to,
                                         self.workspace.data_ptr(), self.workspace.numel(), st)

    def clip(self, max_norm: float, norms: torch.Tensor | None = None, eps: float = 1e-6,
             nonfinite: int = CLIP_PROPAGATE, stream=None):
        """Every client's tensors times min(1, max_norm / (norm + eps)), written to the outputs; the norms where `norms` is
        given.  `nonfinite`: CLIP_ZERO gives zeros for a client whose norm is not finite."""
        _check(self.clip_status(max_norm, norms, eps, nonfinite, stream), "brace_gradient_clip")
