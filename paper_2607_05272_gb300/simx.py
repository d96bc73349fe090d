"""Thin ctypes binding of libsimx.so (include/simx.h): argument marshalling only.

Every step of the rollout, returns, baseline and loss computation runs in the CUDA
library; this module turns torch tensors and dicts into the C structs and pointers
the ABI takes, and raises ``SimxError`` for a non-OK status.  There is no CPU
fallback: if the library is missing the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import threading

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libsimx.so")
_lock = threading.Lock()
_lib = None

OK, EINVAL, ENOMEM, ECUDA, EOVERFLOW, ESTATE = range(6)
POLICY = {"sample": 0, "argmax": 1, "static": 2, "rr": 3, "sq": 4, "random": 5, "external": 6}
ALGO = {"reinforce": 0, "ppo": 1}
TRACE_WIDTH = 4
MAX_LAYERS = 6  # SIMX_MAX_LAYERS
STATE_HEADER_WORDS = 32


class SimxError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("simx status %d: %s" % (status, msg))
        self.status = status


class Config(C.Structure):
    _fields_ = [
        ("abi_version", C.c_uint32), ("mode", C.c_uint32), ("n_envs", C.c_uint32),
        ("n_servers", C.c_uint32), ("n_types", C.c_uint32), ("queue_cap", C.c_uint32),
        ("episode_len", C.c_uint32), ("arrival_kind", C.c_uint32),
        ("cand_mean_gap_us", C.c_float), ("n_mod_states", C.c_uint32),
        ("accept_thr", C.c_uint32 * 2), ("dwell_mean_us", C.c_float),
        ("epoch_us", C.c_uint32), ("diurnal_len", C.c_uint32),
        ("diurnal_rate", C.c_float * 128), ("burst_sigma", C.c_float),
        ("type0_thr", C.c_uint32), ("alpha_us", C.c_uint32 * 2), ("beta_us", C.c_uint32 * 2),
        ("cost_type", C.c_int32), ("cost_kind", C.c_uint32), ("cost_scale_us", C.c_float),
        ("pareto_inv_alpha", C.c_float), ("w_wait", C.c_float * 2), ("n_bsizes", C.c_uint32),
        ("bsizes", C.c_uint32 * 8), ("static_bi", C.c_uint32), ("obs_extra", C.c_uint32),
        ("obs_dim", C.c_uint32), ("t_window_us", C.c_float), ("rate_scale", C.c_float),
        ("rate_ref", C.c_float), ("busy_norm_us", C.c_float), ("phase_period_us", C.c_uint32),
        ("dwell_kind", C.c_uint32), ("srv_speed16", C.c_uint32 * 8),
        ("action_layout", C.c_uint32),
    ]


class Mlp(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("dims", C.c_int32 * (MAX_LAYERS + 1)),
                ("W", C.c_void_p * MAX_LAYERS), ("b", C.c_void_p * MAX_LAYERS),
                ("has_value", C.c_int32), ("act", C.c_int32 * MAX_LAYERS),
                ("grid", C.c_int32), ("gx", C.c_int32 * MAX_LAYERS)]


ACT = {"tanh": 0, "identity": 1, "gelu": 2}


class Rollout(C.Structure):
    _fields_ = [("ld", C.c_int64), ("obs", C.c_void_p), ("action", C.c_void_p),
                ("logp", C.c_void_p), ("value", C.c_void_p), ("reward", C.c_void_p),
                ("done", C.c_void_p), ("trace", C.c_void_p)]


class LossParams(C.Structure):
    _fields_ = [("algo", C.c_int32), ("clip_eps", C.c_float), ("c_value", C.c_float),
                ("c_entropy", C.c_float), ("precision", C.c_int32)]


PRECISION = {"fp32": 0, "tf32": 1}


class Counters(C.Structure):
    _fields_ = [("arrived", C.c_uint64), ("dropped", C.c_uint64), ("dispatched", C.c_uint64),
                ("batches", C.c_uint64), ("queued", C.c_uint64), ("sum_wait_us", C.c_uint64),
                ("decisions", C.c_uint64), ("envs_flagged", C.c_uint32), ("status_or", C.c_uint32)]


class Logits(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("grad", C.c_void_p), ("ld", C.c_int64),
                ("grad_ld", C.c_int64), ("n", C.c_int64), ("vocab", C.c_int64),
                ("dtype", C.c_int32), ("temperature", C.c_float)]


class TokenLoss(C.Structure):
    _fields_ = [("action", C.c_void_p), ("adv", C.c_void_p), ("logp_old", C.c_void_p),
                ("logp_ref", C.c_void_p), ("weight", C.c_void_p), ("clip_low", C.c_float),
                ("clip_high", C.c_float), ("c_kl", C.c_float), ("c_entropy", C.c_float),
                ("logp", C.c_void_p), ("entropy", C.c_void_p), ("stats", C.c_void_p)]


class PreferenceLoss(C.Structure):
    _fields_ = [("token", C.c_void_p), ("seq_start", C.c_void_p), ("mask", C.c_void_p),
                ("logp_ref", C.c_void_p), ("weight", C.c_void_p), ("pairs", C.c_int64),
                ("beta", C.c_float), ("label_smoothing", C.c_float), ("ratio", C.c_void_p),
                ("margin", C.c_void_p), ("stats", C.c_void_p)]


class Seq(C.Structure):
    _fields_ = [("p", C.c_void_p), ("sb", C.c_int64), ("st", C.c_int64)]


class Scan(C.Structure):
    _fields_ = [("batch", C.c_int64), ("len", C.c_int64), ("channels", C.c_int64),
                ("dtype", C.c_int32), ("x", Seq), ("gate", Seq), ("h", Seq), ("bias", C.c_void_p),
                ("h0", C.c_void_p), ("done", C.c_void_p), ("done_sb", C.c_int64),
                ("done_st", C.c_int64), ("h_last", C.c_void_p), ("dh", Seq), ("dx", Seq),
                ("dgate", Seq), ("dh_last", C.c_void_p), ("dbias", C.c_void_p),
                ("dh0", C.c_void_p)]


class Norm(C.Structure):
    _fields_ = [("n", C.c_int64), ("width", C.c_int64), ("dtype", C.c_int32), ("p", C.c_float),
                ("eps", C.c_float), ("seed", C.c_uint64), ("step", C.c_uint32),
                ("row_base", C.c_uint32), ("gain", C.c_void_p), ("rstd", C.c_void_p),
                ("x", C.c_void_p), ("x_ld", C.c_int64), ("residual", C.c_void_p),
                ("residual_ld", C.c_int64), ("z", C.c_void_p), ("z_ld", C.c_int64),
                ("y", C.c_void_p), ("y_ld", C.c_int64), ("dy", C.c_void_p), ("dy_ld", C.c_int64),
                ("dz", C.c_void_p), ("dz_ld", C.c_int64), ("dx", C.c_void_p), ("dx_ld", C.c_int64),
                ("dresidual", C.c_void_p), ("dresidual_ld", C.c_int64), ("dgain", C.c_void_p)]


class Heads(C.Structure):
    _fields_ = [("p", C.c_void_p), ("sb", C.c_int64), ("st", C.c_int64), ("sh", C.c_int64)]


class Attention(C.Structure):
    _fields_ = [("batch", C.c_int64), ("len", C.c_int64), ("heads", C.c_int64), ("kv_heads", C.c_int64),
                ("dk", C.c_int64), ("dv", C.c_int64), ("dtype", C.c_int32), ("scale", C.c_float),
                ("q", Heads), ("k", Heads), ("v", Heads), ("o", Heads), ("log_decay", C.c_void_p),
                ("s0", C.c_void_p), ("done", C.c_void_p), ("done_sb", C.c_int64), ("done_st", C.c_int64),
                ("s_last", C.c_void_p), ("grad_o", Heads), ("grad_q", Heads), ("grad_k", Heads),
                ("grad_v", Heads), ("ds_last", C.c_void_p), ("ds0", C.c_void_p)]


class Rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("sn", C.c_int64), ("sh", C.c_int64)]


class HeadNorm(C.Structure):
    _fields_ = [("n", C.c_int64), ("q_heads", C.c_int64), ("k_heads", C.c_int64), ("dim", C.c_int64),
                ("pairs", C.c_int64), ("dtype", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_float),
                ("position", C.c_void_p), ("turns", C.c_void_p), ("q_gain", C.c_void_p),
                ("k_gain", C.c_void_p), ("q", Rows), ("k", Rows), ("q_out", Rows), ("k_out", Rows),
                ("dq", Rows), ("dk", Rows), ("dq_gain", C.c_void_p), ("dk_gain", C.c_void_p)]


class Logprobs(C.Structure):
    _fields_ = [("token", C.c_void_p), ("logp", C.c_void_p), ("entropy", C.c_void_p),
                ("top_logp", C.c_void_p), ("top_index", C.c_void_p), ("top", C.c_int64)]


# (name, restype, argtypes) of every exported function, in header order.
P, I32, I64, U32, U64, F, SZ = (C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_uint64,
                                C.c_float, C.c_size_t)
SIGNATURES = [
    ("simx_obs_dim", U32, [P]),
    ("simx_state_words", U64, [P]),
    ("sim_create", C.c_int, [P, C.c_int, P]),
    ("sim_destroy", None, [P]),
    ("sim_reset", C.c_int, [P, U64, P]),
    ("sim_set_trace", C.c_int, [P, P, P, P, U32]),
    ("simx_adam_workspace_size", SZ, [I64]),
    ("simx_adam_step", C.c_int, [P, P, P, P, P, I64, I64, P, P, P, SZ, P]),
    ("sim_observe", C.c_int, [P, P, I64, P]),
    ("sim_step_batched", C.c_int, [P, P, P, C.c_int, P, I64, P, P, P, P, P]),
    ("rollout_collect", C.c_int, [P, P, C.c_int, I32, P, P]),
    ("simx_launch_shape", C.c_int, [P, P, C.c_int, P]),
    ("simx_rollout_kernel", C.c_int, [P, P, C.c_int, P]),
    ("simx_forward_columns", C.c_int32, [P, I64]),
    ("simx_loss_kernel", C.c_int32, [P, I64, C.c_int]),
    ("policy_forward", C.c_int, [P, P, I64, I64, C.c_int, U64, U32, U32, P, P, P, P, P]),
    ("policy_forward_workspace_size", SZ, [P]),
    ("policy_forward_ws", C.c_int, [P, P, I64, I64, C.c_int, U64, U32, U32, P, P, P, P, P, SZ, P]),
    ("compute_returns_gae", C.c_int, [P, P, P, P, I64, I64, I64, F, F, P, P, P]),
    ("returns_baseline_workspace_size", SZ, [I64]),
    ("returns_baseline", C.c_int, [P, I64, P, P, P, SZ, P]),
    ("ppo_loss_grad_workspace_size", SZ, [P, I64]),
    ("ppo_loss_grad", C.c_int, [P, P, I64, P, P, P, I64, P, P, P, P, SZ, P]),
    ("ppo_loss_grad_noalloc", C.c_int, [P, P, I64, P, P, P, I64, P, P, P, P]),
    ("simx_token_loss_grad_workspace_size", SZ, [I64]),
    ("simx_token_loss_grad", C.c_int, [P, P, P, SZ, P]),
    ("simx_preference_loss_grad_workspace_size", SZ, [I64, I64]),
    ("simx_preference_loss_grad", C.c_int, [P, P, P, SZ, P]),
    ("simx_gated_scan_workspace_size", SZ, [I64, I64, I64]),
    ("simx_gated_scan", C.c_int, [P, P, SZ, P]),
    ("simx_gated_scan_grad", C.c_int, [P, P, SZ, P]),
    ("simx_dropout_add_norm", C.c_int, [P, P]),
    ("simx_dropout_add_norm_grad_workspace_size", SZ, [I64, I64]),
    ("simx_dropout_add_norm_grad", C.c_int, [P, P, SZ, P]),
    ("simx_decay_attention_workspace_size", SZ, [I64] * 6),
    ("simx_decay_attention", C.c_int, [P, P, SZ, P]),
    ("simx_decay_attention_grad_workspace_size", SZ, [I64] * 6),
    ("simx_decay_attention_grad", C.c_int, [P, P, SZ, P]),
    ("simx_head_norm_rotate", C.c_int, [P, P]),
    ("simx_head_norm_rotate_grad_workspace_size", SZ, [I64] * 4),
    ("simx_head_norm_rotate_grad", C.c_int, [P, P, SZ, P]),
    ("simx_token_logprobs", C.c_int, [P, P, P]),
    ("sim_stats", C.c_int, [P, P]),
    ("sim_save", C.c_int, [P, P, U64]),
    ("sim_load", C.c_int, [P, P, U64]),
    ("simx_last_status", C.c_int, [P, P]),
    ("simx_launches", U64, []),
    ("simx_fma_probe", C.c_int, [I64, P, P, P]),
    ("simx_fma_probe_sink_floats", SZ, []),
    ("simx_math_check", C.c_int, [C.c_int, P, P]),
    ("simx_strerror", C.c_char_p, [C.c_int]),
    ("simx_last_error", C.c_char_p, []),
]


def lib():
    """Load libsimx.so (built by build.py); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError("libsimx.so is not built (%s); run "
                                   "paper_2607_05272_gb300.build.build()" % LIB_PATH)
            L = C.CDLL(LIB_PATH)
            for name, res, args in SIGNATURES:
                fn = getattr(L, name)
                fn.restype = res
                fn.argtypes = args
            _lib = L
    return _lib


def _check(status: int):
    if status != OK:
        raise SimxError(status, lib().simx_last_error().decode())


def make_config(cfg: dict) -> Config:
    c = Config()
    for name, _ in Config._fields_:
        v = cfg[name]
        if isinstance(v, (list, tuple)):
            arr = getattr(c, name)
            for i, x in enumerate(v):
                arr[i] = x
        else:
            setattr(c, name, v)
    return c


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is not None:
        return C.c_void_p(stream)
    import torch
    # the handle alone, where torch gives it: current_stream() builds an object, 2.8 us of a call
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is not None:
        return C.c_void_p(raw(torch.cuda.current_device()))
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


class Policy:
    """A simx_mlp over device tensors W_l [out, in] and b_l [out] (fp32, contiguous);
    acts: the activation after each hidden layer ("tanh", "identity" or "gelu"; default
    tanh); grid: for a grid policy (the exact policy forward), the input grid exponent of
    every layer (its weights must lie on the grid that workloads.grid_check checks)."""

    def __init__(self, Ws, bs, has_value: bool, acts=None, grid=None):
        self.Ws = [w.contiguous() for w in Ws]
        self.bs = [b.contiguous() for b in bs]
        self.has_value = bool(has_value)
        m = Mlp()
        m.n_layers = len(self.Ws)
        m.dims[0] = self.Ws[0].shape[1]
        for l, w in enumerate(self.Ws):
            assert w.dtype.is_floating_point and w.is_cuda
            m.dims[l + 1] = w.shape[0]
            m.W[l] = w.data_ptr()
            m.b[l] = self.bs[l].data_ptr()
        m.has_value = int(self.has_value)
        for l, a in enumerate(acts or []):
            m.act[l] = ACT[a] if isinstance(a, str) else int(a)
        if grid is not None:
            m.grid = 1
            for l, e in enumerate(grid):
                m.gx[l] = int(e)
        self.c = m

    flat = None  # the flat parameter vector when built by from_flat

    @classmethod
    def from_flat(cls, flat, dims, has_value: bool, acts=None, grid=None):
        """A policy whose W_l, b_l are views into one flat fp32 device vector in the
        gradient's order (W0, b0, W1, b1, ...): the optimiser updates it in place."""
        Ws, bs, off = [], [], 0
        for k, n in zip(dims[:-1], dims[1:]):
            Ws.append(flat[off:off + n * k].view(n, k))
            off += n * k
            bs.append(flat[off:off + n])
            off += n
        assert off == flat.numel()
        pol = cls(Ws, bs, has_value, acts, grid)
        pol.flat = flat
        return pol

    @property
    def n_actions(self) -> int:
        return self.Ws[-1].shape[0] - (1 if self.has_value else 0)

    @property
    def n_params(self) -> int:
        return sum(w.numel() + b.numel() for w, b in zip(self.Ws, self.bs))


def launches() -> int:
    """Kernels the library has launched so far in this process."""
    return lib().simx_launches()


def obs_dim(cfg: dict) -> int:
    c = make_config(cfg)
    return lib().simx_obs_dim(C.byref(c))


def state_words(cfg: dict) -> int:
    c = make_config(cfg)
    return lib().simx_state_words(C.byref(c))


class Sim:
    """A simulator context (sim_create / sim_destroy)."""

    def __init__(self, cfg: dict, device: int = 0):
        self.cfg = dict(cfg)
        self._c = make_config(cfg)
        h = C.c_void_p()
        _check(lib().sim_create(C.byref(self._c), device, C.byref(h)))
        self._h = h
        self.E = cfg["n_envs"]
        self.D = obs_dim(cfg)
        self.words = state_words(cfg)
        self._trace = None
        if cfg.get("trace") is not None:
            self.set_trace(*cfg["trace"])

    def set_trace(self, gap_us, type=None, cost_us=None):
        """Trace replay input (sim_set_trace): per-request gaps in us, types and costs;
        numpy arrays are copied to the device, device tensors are used as they are
        (int32 / uint8 / int32, values below 2^31).  Takes effect at the next reset."""
        import torch

        def dev(x, dt):
            if x is None:
                return None
            t = x if isinstance(x, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(x).astype(dt))
            return t.contiguous().cuda()
        g = dev(gap_us, np.int32)
        ty = dev(type, np.uint8)
        co = dev(cost_us, np.int32)
        _check(lib().sim_set_trace(self._h, g.data_ptr(), _ptr(ty), _ptr(co), len(g)))
        self._trace = (g, ty, co)

    def close(self):
        if getattr(self, "_h", None):
            lib().sim_destroy(self._h)
            self._h = None

    __del__ = close

    def reset(self, seed: int, stream=None):
        _check(lib().sim_reset(self._h, seed, _stream(stream)))

    def observe(self, obs, stream=None):
        _check(lib().sim_observe(self._h, _ptr(obs), obs.shape[-1], _stream(stream)))

    def step(self, policy_mode: str, policy: Policy = None, actions=None, obs=None, reward=None,
             done=None, action=None, logp=None, stream=None):
        ld = obs.shape[-1] if obs is not None else self.E
        _check(lib().sim_step_batched(
            self._h, _ptr(actions), C.byref(policy.c) if policy else None, POLICY[policy_mode],
            _ptr(obs), ld, _ptr(reward), _ptr(done), _ptr(action), _ptr(logp), _stream(stream)))

    def rollout(self, policy_mode: str, horizon: int, buf: dict, policy: Policy = None,
                stream=None):
        r = Rollout()
        r.ld = buf["reward"].shape[-1]
        for k in ("obs", "action", "logp", "value", "reward", "done", "trace"):
            t = buf.get(k)
            setattr(r, k, None if t is None else t.data_ptr())
        _check(lib().rollout_collect(self._h, C.byref(policy.c) if policy else None,
                                     POLICY[policy_mode], horizon, C.byref(r), _stream(stream)))

    def launch_shape(self, policy_mode: str, policy: Policy = None) -> dict:
        """The launch rollout_collect takes (simx_launch_shape): kernel ("fused" or
        "thread"), lanes per env, threads per block, warp-local policy forward, whether
        a grid policy's forward runs on the tensor cores, and whether the FP32 forward
        stages its weights in shared memory."""
        out = (C.c_int32 * 6)()
        _check(lib().simx_launch_shape(self._h, C.byref(policy.c) if policy else None,
                                       POLICY[policy_mode], out))
        return dict(kernel="thread" if out[0] else "fused", lanes=out[1], threads=out[2],
                    mlp_warp=bool(out[3]), tensor_cores=bool(out[4]), staged=bool(out[5]))

    def rollout_kernel(self, policy_mode: str, policy: Policy = None) -> tuple:
        """Which kernel that launch is (simx_rollout_kernel): ("lanes", "thread", "route" or
        "single", where its forward reads the weights)."""
        out = (C.c_int32 * 2)()
        _check(lib().simx_rollout_kernel(self._h, C.byref(policy.c) if policy else None,
                                         POLICY[policy_mode], out))
        return (("lanes", "thread", "route", "single")[out[0]],
                ("l1", "staged", "streamed", "resident", "tensor_cores")[out[1]])

    def stats(self) -> dict:
        c = Counters()
        _check(lib().sim_stats(self._h, C.byref(c)))
        return {name: getattr(c, name) for name, _ in Counters._fields_}

    def last_status(self) -> tuple:
        code = C.c_uint32()
        st = lib().simx_last_status(self._h, C.byref(code))
        return st, code.value

    def save(self):
        import numpy as np
        out = np.zeros(self.E * self.words, np.uint32)
        _check(lib().sim_save(self._h, out.ctypes.data, out.size))
        return out.reshape(self.E, self.words)

    def load(self, words):
        import numpy as np
        w = np.ascontiguousarray(words, dtype=np.uint32).ravel()
        _check(lib().sim_load(self._h, w.ctypes.data, w.size))


def alloc_rollout(E: int, D: int, H: int, has_value: bool = False, trace: bool = False,
                  device="cuda") -> dict:
    """Device buffers for rollout_collect in the ABI's time-major layouts."""
    import torch
    buf = dict(
        obs=torch.empty((H, D, E), dtype=torch.float32, device=device),
        action=torch.empty((H, E), dtype=torch.uint8, device=device),
        logp=torch.empty((H, E), dtype=torch.float32, device=device),
        reward=torch.empty((H, E), dtype=torch.float32, device=device),
        done=torch.empty((H, E), dtype=torch.uint8, device=device),
    )
    if has_value:
        buf["value"] = torch.empty((H, E), dtype=torch.float32, device=device)
    if trace:
        buf["trace"] = torch.empty((H, TRACE_WIDTH, E), dtype=torch.int64, device=device)
    return buf


def policy_forward_workspace_size(policy: Policy) -> int:
    return lib().policy_forward_workspace_size(C.byref(policy.c))


def policy_forward(policy: Policy, obs, n: int, policy_mode: str, seed: int, step: int,
                   env_base: int = 0, logits=None, value=None, action=None, logp=None,
                   stream=None, workspace=None):
    """policy_forward, or policy_forward_ws when a device workspace (uint8 tensor of
    policy_forward_workspace_size bytes) is given: needed for concurrent streams and for
    CUDA-graph capture."""
    if workspace is None:
        _check(lib().policy_forward(C.byref(policy.c), _ptr(obs), obs.shape[-1], n,
                                    POLICY[policy_mode], seed, step, env_base, _ptr(logits),
                                    _ptr(value), _ptr(action), _ptr(logp), _stream(stream)))
        return
    _check(lib().policy_forward_ws(C.byref(policy.c), _ptr(obs), obs.shape[-1], n,
                                   POLICY[policy_mode], seed, step, env_base, _ptr(logits),
                                   _ptr(value), _ptr(action), _ptr(logp), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)))


def compute_returns_gae(rew, done, gamma: float, lam: float, ret, adv=None, val=None,
                        last_val=None, stream=None):
    T, E = rew.shape[0], rew.shape[1]
    _check(lib().compute_returns_gae(_ptr(rew), _ptr(val), _ptr(done), _ptr(last_val), T, E,
                                     rew.shape[1], gamma, lam, _ptr(ret), _ptr(adv),
                                     _stream(stream)))


def returns_baseline_workspace_size(n: int) -> int:
    return lib().returns_baseline_workspace_size(n)


def returns_baseline(x, adv_out, mean_out, workspace, stream=None):
    _check(lib().returns_baseline(_ptr(x), x.numel(), _ptr(adv_out), _ptr(mean_out),
                                  _ptr(workspace), workspace.numel() * workspace.element_size(),
                                  _stream(stream)))


def ppo_loss_grad_workspace_size(policy: Policy, n: int) -> int:
    return lib().ppo_loss_grad_workspace_size(C.byref(policy.c), n)


def forward_columns(policy: Policy, n: int) -> int:
    """Columns per block of policy_forward's block forward, 0 for its lane-group kernel."""
    return lib().simx_forward_columns(C.byref(policy.c), n)


def loss_kernel(policy: Policy, n: int, precision: str = "fp32") -> str:
    """Which kernel ppo_loss_grad takes for n rows (simx_loss_kernel)."""
    k = lib().simx_loss_kernel(C.byref(policy.c), n, PRECISION[precision])
    return ("gemm", "fused", "block", "tc", "wide")[k] if k >= 0 else "refused"


def ppo_loss_grad(policy: Policy, buf: dict, ret, adv, idx, n: int, algo: str, clip_eps: float,
                  c_value: float, c_entropy: float, grad, stats, workspace, stream=None,
                  precision: str = "fp32"):
    r = Rollout()
    r.ld = buf["action"].shape[-1]
    for k in ("obs", "action", "logp", "value", "reward", "done", "trace"):
        t = buf.get(k)
        setattr(r, k, None if t is None else t.data_ptr())
    p = LossParams(ALGO[algo], clip_eps, c_value, c_entropy, PRECISION[precision])
    _check(lib().ppo_loss_grad(C.byref(policy.c), C.byref(r), r.ld, _ptr(ret), _ptr(adv),
                               _ptr(idx), n, C.byref(p), _ptr(grad), _ptr(stats), _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream(stream)))


class AdamParams(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float),
                ("eps", C.c_float), ("max_grad_norm", C.c_float)]


def adam_workspace_size(n: int) -> int:
    return lib().simx_adam_workspace_size(n)


def adam_step(params, grad, m, v, t, lr: float, beta1: float = 0.9, beta2: float = 0.999,
              eps: float = 1e-8, max_grad_norm: float = 0.0, mask=None, workspace=None,
              stream=None):
    """simx_adam_step on flat fp32 device vectors (mask: uint8 or None).  t: the step
    number (int), or an int64 device tensor of one element that the step increments."""
    p = AdamParams(lr, beta1, beta2, eps, max_grad_norm)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    dev = not isinstance(t, int)
    _check(lib().simx_adam_step(_ptr(params), _ptr(grad), _ptr(m), _ptr(v), _ptr(mask),
                                params.numel(), 0 if dev else t, _ptr(t) if dev else None,
                                C.byref(p), _ptr(workspace), ws_bytes, _stream(stream)))


NOALLOC_SCRATCH_BYTES = 64 << 20


def ppo_loss_grad_noalloc(policy: Policy, buf: dict, ret, adv, idx, n: int, algo: str,
                          clip_eps: float, c_value: float, c_entropy: float, grad, stats,
                          stream=None, precision: str = "fp32"):
    """ppo_loss_grad without a caller workspace: the scratch is a buffer inside the
    library, for callers that cannot allocate device memory (see include/simx.h)."""
    r = Rollout()
    r.ld = buf["action"].shape[-1]
    for k in ("obs", "action", "logp", "value", "reward", "done", "trace"):
        t = buf.get(k)
        setattr(r, k, None if t is None else t.data_ptr())
    p = LossParams(ALGO[algo], clip_eps, c_value, c_entropy, PRECISION[precision])
    _check(lib().ppo_loss_grad_noalloc(C.byref(policy.c), C.byref(r), r.ld, _ptr(ret), _ptr(adv),
                                       _ptr(idx), n, C.byref(p), _ptr(grad), _ptr(stats),
                                       _stream(stream)))


# Operators of sequence policies (include/simx.h has the formulas).  Tensors are fp32 or bf16 and
# strided as they come, with a last axis of unit stride; per-row values, parameters, states and
# statistics are contiguous fp32.

def _refuse(msg: str):
    raise SimxError(EINVAL, msg)


def _image(cls):
    """A function from a structure's fields, in order and nested ones flattened, to its bytes (pointers
    as integers).  Packing takes a quarter of the time of filling the ctypes structure."""
    def codes(c):
        return "".join(codes(f[1]) if issubclass(f[1], C.Structure) else f[1]._type_ for f in c._fields_)
    # "l" and "L" of ctypes' 64-bit integers are 64 bits in native layout too
    layout = struct.Struct("@" + codes(cls) + "0q")
    assert layout.size == C.sizeof(cls)
    pack = layout.pack

    def image(*values):
        try:
            return pack(*values)
        except (struct.error, OverflowError) as e:
            _refuse("argument out of range: %s" % e)
    return image


_logits_image, _token_loss_image = _image(Logits), _image(TokenLoss)
_preference_loss_image, _scan_image, _norm_image = _image(PreferenceLoss), _image(Scan), _image(Norm)


def _tensor(t, name: str, like, shape, dev: int):
    """A data tensor: `like`'s dtype, `shape`, on device `dev`, unit stride along the last axis."""
    if t is None:
        return 0
    if t.dtype is not like.dtype or t.shape != shape or t.get_device() != dev:
        _refuse("%s: %s %s on %s expected, got %s %s on %s" % (
            name, tuple(shape), like.dtype, like.device, tuple(t.shape), t.dtype, t.device))
    if not t.is_contiguous() and t.stride(-1) != 1 and t.shape[-1] > 1:
        _refuse("%s: the last axis needs unit stride" % name)
    return t.data_ptr()


def _flat(t, name: str, dtype, shape, dev: int):
    """A contiguous tensor of `dtype` and `shape` on device `dev`."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _refuse("%s: contiguous %s %s on cuda:%d expected, got %s %s on %s" % (
            name, tuple(shape), dtype, dev, tuple(t.shape), t.dtype, t.device))
    return t.data_ptr()


def _dtype(t, name: str, ndim: int):
    """(torch, dtype code, shape, device index) of an operator's leading tensor."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dim() != ndim:
        _refuse("%s: a tensor of %d axes expected" % (name, ndim))
    if not t.is_cuda:
        _refuse("%s: not on a CUDA device" % name)
    dev = t.get_device()
    if dev != torch.cuda.current_device():
        _refuse("%s: on %s, which is not the current device" % (name, t.device))
    if t.dtype is torch.float32:
        return torch, 0, t.shape, dev
    if t.dtype is torch.bfloat16:
        return torch, 1, t.shape, dev
    _refuse("%s: float32 or bfloat16 expected, got %s" % (name, t.dtype))


def _workspace(ws, dev: int):
    """(pointer, bytes) of a workspace tensor or None."""
    if ws is None:
        return None, 0
    if ws.get_device() != dev or not ws.is_contiguous():
        _refuse("workspace: a contiguous tensor on cuda:%d expected" % dev)
    return ws.data_ptr(), ws.nbytes


def _ld(t, shape) -> int:
    """Row stride of a [n, width] tensor (a single row has none)."""
    return t.stride(0) if shape[0] > 1 else shape[1]


def _logits(logits, grad, temperature):
    torch, dt, shape, dev = _dtype(logits, "logits", 2)
    n, vocab = shape
    return torch, dev, n, _logits_image(_tensor(logits, "logits", logits, shape, dev),
                                        _tensor(grad, "grad", logits, shape, dev),
                                        _ld(logits, shape), _ld(grad, shape) if grad is not None else 0,
                                        n, vocab, dt, temperature)


def token_loss_grad_workspace_size(n: int) -> int:
    return lib().simx_token_loss_grad_workspace_size(n)


def token_loss_grad(logits, action, adv, stats, workspace, logp_old=None, logp_ref=None,
                    weight=None, clip_low: float = 0.2, clip_high: float = 0.2, c_kl: float = 0.0,
                    c_entropy: float = 0.0, temperature: float = 1.0, grad=None, logp=None,
                    entropy=None, stream=None):
    """The clipped policy loss with KL and entropy terms from logits [n, vocab], and its gradient
    with respect to them (simx_token_loss_grad).  action: int64 [n]; adv, logp_old, logp_ref,
    weight, logp, entropy: fp32 [n] or None; stats: fp32 [5] = loss, policy term, KL, entropy,
    clipped share; grad: like logits, logits itself, or None."""
    torch, dev, n, x = _logits(logits, grad, temperature)
    n, f = (n,), torch.float32
    a = _token_loss_image(
        _flat(action, "action", torch.int64, n, dev), _flat(adv, "adv", f, n, dev),
        _flat(logp_old, "logp_old", f, n, dev), _flat(logp_ref, "logp_ref", f, n, dev),
        _flat(weight, "weight", f, n, dev), clip_low, clip_high, c_kl, c_entropy,
        _flat(logp, "logp", f, n, dev), _flat(entropy, "entropy", f, n, dev),
        _flat(stats, "stats", f, (5,), dev))
    _check(lib().simx_token_loss_grad(x, a, *_workspace(workspace, dev), _stream(stream)))


def preference_loss_grad_workspace_size(n: int, pairs: int) -> int:
    return lib().simx_preference_loss_grad_workspace_size(n, pairs)


def preference_loss_grad(logits, token, seq_start, stats, workspace, logp_ref=None, mask=None,
                         weight=None, beta: float = 0.1, label_smoothing: float = 0.0,
                         temperature: float = 1.0, grad=None, ratio=None, margin=None, stream=None):
    """The preference loss on pairs of sequences from their packed logits [n, vocab], and its
    gradient with respect to them (simx_preference_loss_grad).  token: int64 [n]; seq_start: int64
    [2 * pairs + 1] row offsets, the preferred sequence of a pair first; mask: uint8 [n] or None;
    logp_ref: fp32 [n] or None; weight, margin: fp32 [pairs] or None; ratio: fp32 [2 * pairs] or
    None; stats: fp32 [3] = loss, share of pairs in the right order, mean margin."""
    torch, dev, n, x = _logits(logits, grad, temperature)
    n, f = (n,), torch.float32
    if seq_start is None or seq_start.dim() != 1 or len(seq_start) % 2 != 1:
        _refuse("seq_start: 2 * pairs + 1 row offsets expected")
    pairs = len(seq_start) // 2
    a = _preference_loss_image(
        _flat(token, "token", torch.int64, n, dev),
        _flat(seq_start, "seq_start", torch.int64, seq_start.shape, dev),
        _flat(mask, "mask", torch.uint8, n, dev), _flat(logp_ref, "logp_ref", f, n, dev),
        _flat(weight, "weight", f, (pairs,), dev), pairs, beta, label_smoothing,
        _flat(ratio, "ratio", f, (2 * pairs,), dev), _flat(margin, "margin", f, (pairs,), dev),
        _flat(stats, "stats", f, (3,), dev))
    _check(lib().simx_preference_loss_grad(x, a, *_workspace(workspace, dev), _stream(stream)))


def gated_scan_workspace_size(batch: int, length: int, channels: int) -> int:
    return lib().simx_gated_scan_workspace_size(batch, length, channels)


def _seq(t, name: str, like, shape, dev: int):
    """The fields of a Seq of a tensor of `like`'s dtype."""
    p = _tensor(t, name, like, shape, dev)
    if t is None:
        return 0, 0, 0
    sb, st, _ = t.stride()
    return p, sb, st


def _scan(x, gate, h, bias, h0, done):
    """Shape and device of a scan, and the fields of its Scan before h_last."""
    torch, dt, shape, dev = _dtype(x, "x", 3)
    b, t, c = shape
    d, dsb, dst = 0, 0, 0
    if done is not None:
        if done.dtype is not torch.uint8 or done.shape != (b, t) or done.get_device() != dev:
            _refuse("done: uint8 %s on cuda:%d expected" % ((b, t), dev))
        d = done.data_ptr()
        dsb, dst = done.stride()
    f = torch.float32
    return f, shape, dev, (b, t, c, dt, *_seq(x, "x", x, shape, dev),
                           *_seq(gate, "gate", x, shape, dev), *_seq(h, "h", x, shape, dev),
                           _flat(bias, "bias", f, (c,), dev), _flat(h0, "h0", f, (b, c), dev),
                           d, dsb, dst)


def gated_scan(x, gate, h, workspace=None, bias=None, h0=None, done=None, h_last=None, stream=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a_t = sigmoid(gate_t + bias) over x, gate, h
    [batch, len, channels] of any batch and time strides (simx_gated_scan).  bias: fp32 [channels];
    h0, h_last: fp32 [batch, channels] (h_last may be h0: the single-token step of serving); done:
    uint8 [batch, len], nonzero where the state is not carried on; each of them may be None."""
    f, (b, _, c), dev, head = _scan(x, gate, h, bias, h0, done)
    s = _scan_image(*head, _flat(h_last, "h_last", f, (b, c), dev), *(0,) * 12)
    _check(lib().simx_gated_scan(s, *_workspace(workspace, dev), _stream(stream)))


def gated_scan_grad(x, gate, h, dh, dx, dgate, workspace, bias=None, h0=None, done=None,
                    dh_last=None, dbias=None, dh0=None, stream=None):
    """The backward pass of gated_scan (simx_gated_scan_grad): dx, dgate and, where given, dbias
    and dh0 from dh and dh_last, with h as the forward pass left it."""
    f, shape, dev, head = _scan(x, gate, h, bias, h0, done)
    state = (shape[0], shape[2])
    s = _scan_image(*head, 0, *_seq(dh, "dh", x, shape, dev), *_seq(dx, "dx", x, shape, dev),
                    *_seq(dgate, "dgate", x, shape, dev), _flat(dh_last, "dh_last", f, state, dev),
                    _flat(dbias, "dbias", f, state[1:], dev), _flat(dh0, "dh0", f, state, dev))
    _check(lib().simx_gated_scan_grad(s, *_workspace(workspace, dev), _stream(stream)))


def _rows(t, name: str, like, shape, dev: int):
    """(pointer, row stride) of a tensor of `like`'s dtype."""
    return (_tensor(t, name, like, shape, dev), _ld(t, shape)) if t is not None else (0, 0)


def _norm(like, name: str, gain, rstd, p, eps, seed, step, row_base):
    torch, dt, shape, dev = _dtype(like, name, 2)
    n, width = shape
    if not (0 <= seed < 1 << 64 and 0 <= step < 1 << 32 and 0 <= row_base < 1 << 32):
        _refuse("seed, step or row_base out of range")
    f = torch.float32
    return f, shape, dev, (n, width, dt, p, eps, seed, step, row_base,
                           _flat(gain, "gain", f, (width,), dev), _flat(rstd, "rstd", f, (n,), dev))


def dropout_add_norm(x, gain, y, residual=None, z=None, rstd=None, p: float = 0.0,
                     eps: float = 1e-6, seed: int = 0, step: int = 0, row_base: int = 0,
                     stream=None):
    """z = residual + dropout_p(x) and y = rms_norm(z) * gain over rows [n, width]
    (simx_dropout_add_norm).  The mask is a function of (seed, step, row_base + row, column) and is
    not stored.  gain: fp32 [width]; rstd: fp32 [n] or None, kept for the backward pass."""
    _, n, dev, head = _norm(x, "x", gain, rstd, p, eps, seed, step, row_base)
    a = _norm_image(*head, *_rows(x, "x", x, n, dev), *_rows(residual, "residual", x, n, dev),
                    *_rows(z, "z", x, n, dev), *_rows(y, "y", x, n, dev), *(0,) * 9)
    _check(lib().simx_dropout_add_norm(a, _stream(stream)))


def dropout_add_norm_grad_workspace_size(n: int, width: int) -> int:
    return lib().simx_dropout_add_norm_grad_workspace_size(n, width)


def dropout_add_norm_grad(z, gain, rstd, dy, dx, workspace, dz=None, dresidual=None, dgain=None,
                          p: float = 0.0, seed: int = 0, step: int = 0, row_base: int = 0,
                          stream=None):
    """The backward pass of dropout_add_norm (simx_dropout_add_norm_grad): dx, dresidual and dgain
    (each may be None) from dy and dz, with z and rstd as the forward pass left them and the same
    p, seed, step and row_base."""
    f, n, dev, head = _norm(z, "z", gain, rstd, p, 0.0, seed, step, row_base)
    a = _norm_image(*head, 0, 0, 0, 0, *_rows(z, "z", z, n, dev), 0, 0, *_rows(dy, "dy", z, n, dev),
                    *_rows(dz, "dz", z, n, dev), *_rows(dx, "dx", z, n, dev),
                    *_rows(dresidual, "dresidual", z, n, dev), _flat(dgain, "dgain", f, n[1:], dev))
    _check(lib().simx_dropout_add_norm_grad(a, *_workspace(workspace, dev), _stream(stream)))


# Operators of attention policies (include/simx.h has the formulas).

_attention_image, _head_norm_image, _logprobs_image = _image(Attention), _image(HeadNorm), _image(Logprobs)


def _heads(t, name: str, like, shape, dev: int):
    """The fields of a Heads of a tensor [batch, len, heads, dim] of `like`'s dtype."""
    p = _tensor(t, name, like, shape, dev)
    if t is None:
        return 0, 0, 0, 0
    sb, st, sh, _ = t.stride()
    return p, sb, st, sh


def _attention(q, k, v, log_decay, scale, s0, done):
    """Shapes and device of an attention, and the fields of its Attention: before o, and from log_decay to
    before s_last."""
    torch, dt, shape, dev = _dtype(q, "q", 4)
    b, t, h, dk = shape
    if k is None or v is None or k.dim() != 4 or v.dim() != 4:
        _refuse("k, v: tensors of 4 axes expected")
    hk, dv = k.shape[2], v.shape[3]
    d, dsb, dst = 0, 0, 0
    if done is not None:
        if done.dtype is not torch.uint8 or done.shape != (b, t) or done.get_device() != dev:
            _refuse("done: uint8 %s on cuda:%d expected" % ((b, t), dev))
        d = done.data_ptr()
        dsb, dst = done.stride()
    f, state = torch.float32, (b, h, dk, dv)
    return f, state, (b, t, h, dv), dev, (
        b, t, h, hk, dk, dv, dt, max(dk, 1) ** -0.5 if scale is None else scale, *_heads(q, "q", q, shape, dev),
        *_heads(k, "k", q, (b, t, hk, dk), dev), *_heads(v, "v", q, (b, t, hk, dv), dev)), (
        _flat(log_decay, "log_decay", f, (h,), dev), _flat(s0, "s0", f, state, dev), d, dsb, dst)


def decay_attention_workspace_size(batch: int, length: int, heads: int, kv_heads: int, dk: int, dv: int) -> int:
    return lib().simx_decay_attention_workspace_size(batch, length, heads, kv_heads, dk, dv)


def decay_attention(q, k, v, o, log_decay, workspace=None, scale=None, s0=None, done=None, s_last=None,
                    stream=None):
    """Linear attention with a decay for each head, S_t = e^log_decay S_{t-1} + k_t^T v_t and
    o_t = scale q_t S_t (simx_decay_attention).  q [batch, len, heads, dk] and o [.., heads, dv]; k
    [.., kv_heads, dk] and v [.., kv_heads, dv], of any strides but the last.  log_decay: fp32 [heads], at
    most 0; scale: dk ** -0.5 where None; s0, s_last: fp32 [batch, heads, dk, dv] (s_last may be s0: the
    single-token step of serving); done: uint8 [batch, len], nonzero where the state is not carried on;
    workspace: a tensor of decay_attention_workspace_size bytes, where that is not 0."""
    f, state, out, dev, head, tail = _attention(q, k, v, log_decay, scale, s0, done)
    a = _attention_image(*head, *_heads(o, "o", q, out, dev), *tail, _flat(s_last, "s_last", f, state, dev),
                         *(0,) * 18)
    _check(lib().simx_decay_attention(a, *_workspace(workspace, dev), _stream(stream)))


def decay_attention_grad_workspace_size(batch: int, length: int, heads: int, kv_heads: int, dk: int,
                                        dv: int) -> int:
    return lib().simx_decay_attention_grad_workspace_size(batch, length, heads, kv_heads, dk, dv)


def decay_attention_grad(q, k, v, grad_o, grad_q, grad_k, grad_v, log_decay, workspace, scale=None, s0=None,
                         done=None, ds_last=None, ds0=None, stream=None):
    """The backward pass of decay_attention (simx_decay_attention_grad): grad_q, grad_k, grad_v and, where
    given, ds0 from grad_o and ds_last."""
    f, state, out, dev, head, tail = _attention(q, k, v, log_decay, scale, s0, done)
    a = _attention_image(*head, 0, 0, 0, 0, *tail, 0, *_heads(grad_o, "grad_o", q, out, dev),
                         *_heads(grad_q, "grad_q", q, q.shape, dev), *_heads(grad_k, "grad_k", q, k.shape, dev),
                         *_heads(grad_v, "grad_v", q, v.shape, dev), _flat(ds_last, "ds_last", f, state, dev),
                         _flat(ds0, "ds0", f, state, dev))
    _check(lib().simx_decay_attention_grad(a, *_workspace(workspace, dev), _stream(stream)))


def rotary_turns(rotated: int, base: float = 10000.0, device="cuda"):
    """The table `turns` of head_norm_rotate for `rotated` elements of a head: pair j turns by
    base ** (-2 j / rotated) radians a position, as int64 [rotated / 2] fractions of a turn in units of
    2^-64."""
    import math

    import torch
    if rotated < 0 or rotated % 2 or not base > 0:
        _refuse("rotated: an even number of elements, base: a positive one expected")
    t = [round(base ** (-2 * j / rotated) / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for j in range(rotated // 2)]
    return torch.tensor([v - 2 ** 64 if v >= 2 ** 63 else v for v in t], dtype=torch.int64, device=device)


def _head_rows(t, name: str, like, shape, dev: int):
    """The fields of a Rows of a tensor [n, heads, dim] of `like`'s dtype."""
    p = _tensor(t, name, like, shape, dev)
    if t is None:
        return 0, 0, 0
    sn, sh, _ = t.stride()
    return p, sn, sh


def _head_norm(q, k, position, turns, q_gain, k_gain, eps, interleaved):
    torch, dt, shape, dev = _dtype(q, "q", 3)
    n, hq, d = shape
    if k is not None and k.dim() != 3:
        _refuse("k: a tensor of 3 axes expected")
    k_shape = (n, 0 if k is None else k.shape[1], d)
    if (position is None) != (turns is None) or (turns is not None and turns.dim() != 1):
        _refuse("position and turns: [n] and [pairs], or neither")
    pairs, f = 0 if turns is None else len(turns), torch.float32
    return f, k_shape, dev, (
        n, hq, k_shape[1], d, pairs, dt, int(interleaved), eps, _flat(position, "position", torch.int64, (n,), dev),
        _flat(turns, "turns", torch.int64, (pairs,), dev), _flat(q_gain, "q_gain", f, (d,), dev),
        _flat(k_gain, "k_gain", f, (d,), dev), *_head_rows(q, "q", q, shape, dev), *_head_rows(k, "k", q, k_shape, dev))


def head_norm_rotate(q, q_out, k=None, k_out=None, position=None, turns=None, q_gain=None, k_gain=None,
                     eps: float = 1e-6, interleaved: bool = False, stream=None):
    """Root-mean-square norm of each head of q [n, heads, dim] and k [n, k_heads, dim], of any token and
    head strides, and the rotation of their pairs by position in the same pass (simx_head_norm_rotate).
    position: int64 [n]; turns: int64 [pairs] as rotary_turns makes it; both None: no rotation; q_gain,
    k_gain: fp32 [dim] or None (ones).  q_out may be q itself, k_out k."""
    _, k_shape, dev, head = _head_norm(q, k, position, turns, q_gain, k_gain, eps, interleaved)
    a = _head_norm_image(*head, *_head_rows(q_out, "q_out", q, q.shape, dev),
                         *_head_rows(k_out, "k_out", q, k_shape, dev), *(0,) * 8)
    _check(lib().simx_head_norm_rotate(a, _stream(stream)))


def head_norm_rotate_grad_workspace_size(n: int, q_heads: int, k_heads: int, dim: int) -> int:
    return lib().simx_head_norm_rotate_grad_workspace_size(n, q_heads, k_heads, dim)


def head_norm_rotate_grad(q, dq_out, dq, k=None, dk_out=None, dk=None, workspace=None, position=None, turns=None,
                          q_gain=None, k_gain=None, dq_gain=None, dk_gain=None, eps: float = 1e-6,
                          interleaved: bool = False, stream=None):
    """The backward pass of head_norm_rotate (simx_head_norm_rotate_grad): dq and dk, and the gains'
    gradients where given (with a workspace), from dq_out and dk_out, with q and k as before the forward
    pass.  dq may be dq_out or q itself, dk dk_out or k."""
    f, k_shape, dev, head = _head_norm(q, k, position, turns, q_gain, k_gain, eps, interleaved)
    gain = k_shape[2:]
    a = _head_norm_image(*head, *_head_rows(dq_out, "dq_out", q, q.shape, dev),
                         *_head_rows(dk_out, "dk_out", q, k_shape, dev), *_head_rows(dq, "dq", q, q.shape, dev),
                         *_head_rows(dk, "dk", q, k_shape, dev), _flat(dq_gain, "dq_gain", f, gain, dev),
                         _flat(dk_gain, "dk_gain", f, gain, dev))
    _check(lib().simx_head_norm_rotate_grad(a, *_workspace(workspace, dev), _stream(stream)))


def token_logprobs(logits, token, logp, entropy=None, top_logp=None, top_index=None, temperature: float = 1.0,
                   stream=None):
    """Log probabilities fp32 [n] of token int64 [n] under logits [n, vocab] (simx_token_logprobs), with
    the entropy fp32 [n] and the most probable tokens of each row: top_index int64 [n, top] and top_logp
    fp32 [n, top], top at most 32, in descending order, the lowest index first among equals.  Each may be
    None."""
    torch, dev, n, x = _logits(logits, None, temperature)
    f = torch.float32
    best = top_logp if top_logp is not None else top_index
    if best is not None and best.dim() != 2:
        _refuse("top_logp, top_index: [n, top] expected")
    top = 0 if best is None else best.shape[1]
    a = _logprobs_image(_flat(token, "token", torch.int64, (n,), dev), _flat(logp, "logp", f, (n,), dev),
                        _flat(entropy, "entropy", f, (n,), dev), _flat(top_logp, "top_logp", f, (n, top), dev),
                        _flat(top_index, "top_index", torch.int64, (n, top), dev), top)
    _check(lib().simx_token_logprobs(x, a, _stream(stream)))


def fma_probe_sink_floats() -> int:
    return lib().simx_fma_probe_sink_floats()


def fma_probe(iters: int, sink, stream=None) -> float:
    """Launch the FP32 FMA-rate probe on the stream; returns the FLOPs it performs."""
    fl = C.c_double(0.0)
    _check(lib().simx_fma_probe(iters, _ptr(sink), C.byref(fl), _stream(stream)))
    return fl.value


def math_check(which: str, count, stream=None):
    """Count into `count` (int64 device tensor of one element) the fp32 inputs on which the
    branch-free "tanh" or "exp" differs from the defining one."""
    _check(lib().simx_math_check({"tanh": 0, "exp": 1}[which], _ptr(count), _stream(stream)))
