"""Python binding of the pe C ABI (include/pe.h): argument marshalling only.

Every step of the path runs in the CUDA kernels of libpe.so.  PyTorch is used
for device memory and streams: tensors are passed to the library as raw
device pointers together with the current CUDA stream.  There is no CPU
fallback: if libpe.so is missing or fails to load, every entry point raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Dict, Optional, Sequence

import torch

from . import workloads as W

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libpe.so")
_lib = None

PE_OK, PE_EINVAL, PE_ENOMEM, PE_ECUDA, PE_EOVERFLOW, PE_ETIMEOUT, PE_ESTATE = range(7)
PE_F32, PE_BF16, PE_F16, PE_E4M3 = 0, 1, 2, 3
PE_ROLLOUT_DETERMINISTIC = 1
MAX_LEVELS, MAX_CH = 32, 4
(PE_PROF_ROLLOUT, PE_PROF_VALUE, PE_PROF_GAE, PE_PROF_PPO_GRAD, PE_PROF_PPO_REDUCE,
 PE_PROF_PPO_ADAM, PE_PROF_PPO_OTHER, PE_PROF_FLEET_PREP, PE_PROF_FLEET_WINDOWS,
 PE_PROF_MLP_POLICY, PE_PROF_MLP_VALUE, PE_PROF_KV_APPEND, PE_PROF_DECODE_ATTN, PE_PROF_TOKEN_LOGP,
 PE_PROF_TOKEN_LOGP_GRAD, PE_PROF_TREE_ATTN, PE_PROF_KV_MOVE) = range(17)
PE_PROF_KINDS = 17


class PEError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"pe status {status}: {msg}")
        self.status = status


class EnvConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_envs", "n_channels", "trace_len", "n_actions", "obs_kind", "actuator_kind",
        "n_levels", "level_init", "g_min", "g_max", "b_min", "b_max", "b_init",
        "episode_len", "budget_q", "scale_phase_mask", "reward_kind", "reward_window")] + [
        ("r_ok", C.c_float), ("r_viol", C.c_float), ("bonus_coef", C.c_float),
        ("level_scale", (C.c_float * MAX_CH) * MAX_LEVELS),
        ("level_tokens", C.c_float * MAX_LEVELS),
        ("seed", C.c_uint64),
        ("level_samples", C.c_int32 * MAX_LEVELS),
        ("n_families", C.c_int32), ("fam_len", C.c_int32 * 4), ("fam_channels", C.c_int32 * 4),
        ("fam_budget_q", C.c_int32 * 4)]


class Net(C.Structure):
    _fields_ = [("obs_dim", C.c_int32), ("hidden", C.c_int32), ("n_actions", C.c_int32),
                ("dtype", C.c_int32)]


ROLLOUT_FIELDS = ("obs", "obs_last", "act", "logp", "value", "last_value", "reward", "done", "viol",
                  "tokens", "excess", "energy_q", "samples", "q")


class RolloutBuf(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ROLLOUT_FIELDS]


class Rule(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "hi_q", "lo_q", "drop30_q", "climb30_q", "climb10_q")]


class PPOConfig(C.Structure):
    _fields_ = [("epochs", C.c_int32), ("minibatch", C.c_int32)] + [
        (n, C.c_float) for n in ("lr", "clip", "vf_coef", "ent_coef", "max_grad_norm",
                                 "beta1", "beta2", "eps")] + [
        ("seed", C.c_uint64), ("iteration", C.c_uint32)]


class KVCacheDesc(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "table")] + [
        (n, C.c_int64) for n in ("n_pages", "page_stride", "slot_stride", "head_stride", "table_stride")] + [
        (n, C.c_int32) for n in ("n_seqs", "max_pages", "page_size", "n_heads", "head_dim", "dtype")]


class KVTokens(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("pos", "seq", "rot", "q", "q_out", "k", "v")] + [
        (n, C.c_int64) for n in ("n_tokens", "max_pos", "q_token_stride", "q_head_stride", "q_out_token_stride",
                                 "q_out_head_stride", "k_token_stride", "k_head_stride", "v_token_stride",
                                 "v_head_stride")] + [
        (n, C.c_int32) for n in ("n_q_heads", "rot_dim", "interleaved")]


class KVScales(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)] + [
        (n, C.c_int64) for n in ("page_stride", "slot_stride", "head_stride")]


class TreeQueries(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "out", "lse", "lens", "mask")] + [
        (n, C.c_int64) for n in ("q_seq_stride", "q_node_stride", "q_head_stride", "out_seq_stride", "out_node_stride",
                                 "out_head_stride", "mask_stride")] + [
        (n, C.c_int32) for n in ("n_nodes", "n_q_heads", "dtype")]


# the same bytes at once: filling the structure's fields costs four times as much
_KV_TOKENS = struct.Struct("17q3i4x").pack
assert struct.calcsize("17q3i4x") == C.sizeof(KVTokens)
_TREE_QUERIES = struct.Struct("12q3i4x").pack
assert struct.calcsize("12q3i4x") == C.sizeof(TreeQueries)


EXPORTS = (
    "pe_env_create", "pe_env_destroy", "pe_env_state_bytes", "pe_env_save", "pe_env_load",
    "pe_param_count", "pe_rollout_workspace_bytes", "pe_rollout", "pe_value_workspace_bytes",
    "pe_value", "pe_device_check", "pe_gae", "pe_ppo_workspace_bytes",
    "pe_ppo_update", "pe_fleet_workspace_bytes", "pe_fleet_windows", "pe_fleet_windows_noalloc",
    "pe_fleet_stagger_workspace_bytes", "pe_fleet_stagger", "pe_env_set_offsets", "pe_rollout_rule", "pe_rollout_replay", "pe_wait_selftest",
    "pe_dual_ascent", "pe_roof_probe",
    "pe_kv_append", "pe_decode_attn_workspace_bytes", "pe_decode_attn", "pe_token_logp", "pe_token_logp_grad",
    "pe_kv_append_at", "pe_decode_attn8_workspace_bytes", "pe_decode_attn8", "pe_tree_attn_workspace_bytes",
    "pe_tree_attn", "pe_kv_move",
    "pe_profile_enable",
    "pe_profile_read", "pe_profile_kind_name", "pe_last_error")


def lib():
    """Load libpe.so (raises if it is missing)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2608_11226_gb300.build.build()")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32
        sig = {
            "pe_env_create": (i32, [vp, vp, vp, C.POINTER(vp)]),
            "pe_env_destroy": (i32, [vp]),
            "pe_env_state_bytes": (i64, [vp]),
            "pe_env_save": (i32, [vp, vp]),
            "pe_env_load": (i32, [vp, vp]),
            "pe_param_count": (i64, [vp]),
            "pe_rollout_workspace_bytes": (i64, [vp, vp]),
            "pe_rollout": (i32, [vp, vp, vp, i32, u32, C.c_float, i32, vp, vp, i64, vp]),
            "pe_value_workspace_bytes": (i64, [vp]),
            "pe_value": (i32, [vp, vp, vp, i64, vp, vp, i64, vp]),
            "pe_device_check": (i32, [vp]),
            "pe_gae": (i32, [vp, vp, vp, vp, i32, i32, C.c_float, C.c_float, vp, vp, vp]),
            "pe_ppo_workspace_bytes": (i64, [vp, vp, i64]),
            "pe_ppo_update": (i32, [vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp,
                                    i64, vp]),
            "pe_fleet_workspace_bytes": (i64, [i32, i32, i32]),
            "pe_fleet_stagger_workspace_bytes": (i64, [i32, i32, i32, i32]),
            "pe_env_set_offsets": (i32, [vp, vp, vp]),
            "pe_dual_ascent": (i32, [vp, i32, i64, i32, i32, C.c_float, C.c_float, C.c_float, C.c_float,
                                     vp, vp, vp]),
            "pe_rollout_rule": (i32, [vp, vp, i32, u32, C.c_float, i32, vp, vp]),
            "pe_rollout_replay": (i32, [vp, vp, i32, u32, C.c_float, i32, vp, vp]),
            "pe_wait_selftest": (i32, [i32, C.c_int64, vp, vp]),
            "pe_fleet_stagger": (i32, [vp, i32, i32, vp, i32, i32, i32, i32, vp, vp, vp, i64, vp]),
            "pe_fleet_windows": (i32, [vp, i32, i32, vp, i32, vp, i64, i32, vp, i32, i64, vp,
                                       vp, vp, i64, vp]),
            "pe_fleet_windows_noalloc": (i32, [vp, i32, i32, vp, i32, vp, i64, i32, vp, i32, i64,
                                               vp, vp, vp]),
            "pe_roof_probe": (i32, [i32, vp, i64, i64, C.POINTER(C.c_double), C.POINTER(C.c_double), vp]),
            "pe_kv_append": (i32, [vp, vp, vp]),
            "pe_decode_attn_workspace_bytes": (i64, [vp, i32]),
            "pe_decode_attn": (i32, [vp, vp, i64, i64, i32, vp, C.c_float, i32, vp, i64, i64, vp, vp, i64, vp]),
            "pe_token_logp": (i32, [vp, i32, i64, i32, i64, vp, C.c_float, vp, vp, vp, i32, vp, vp, vp]),
            "pe_token_logp_grad": (i32, [vp, i32, i64, i32, i64, vp, C.c_float, vp, vp, vp, vp, vp, i64, vp]),
            "pe_kv_append_at": (i32, [vp, vp, vp, vp, i32, vp]),
            "pe_decode_attn8_workspace_bytes": (i64, [vp, i32]),
            "pe_decode_attn8": (i32, [vp, vp, i32, vp, i64, i64, i32, vp, C.c_float, i32, vp, i64, i64, vp, vp, i64, vp]),
            "pe_tree_attn_workspace_bytes": (i64, [vp, i32, i32]),
            "pe_tree_attn": (i32, [vp, vp, vp, C.c_float, i32, vp, i64, vp]),
            "pe_kv_move": (i32, [vp, vp, vp, i64, vp, i64, i32, vp]),
            "pe_profile_enable": (i32, [i32]),
            "pe_profile_read": (i32, [i32, C.POINTER(C.c_double), C.POINTER(C.c_int64)]),
            "pe_profile_kind_name": (C.c_char_p, [i32]),
            "pe_last_error": (C.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status: int):
    if status != PE_OK:
        raise PEError(status, lib().pe_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def env_config(spec: W.EnvSpec) -> EnvConfig:
    c = EnvConfig()
    for name in ("n_envs", "n_channels", "trace_len", "n_actions", "obs_kind", "actuator_kind",
                 "n_levels", "level_init", "g_min", "g_max", "b_min", "b_max", "b_init",
                 "episode_len", "budget_q", "scale_phase_mask", "reward_kind", "reward_window"):
        setattr(c, name, int(getattr(spec, name)))
    c.r_ok, c.r_viol, c.bonus_coef = spec.r_ok, spec.r_viol, spec.bonus_coef
    for l, row in enumerate(spec.level_scale):
        for ch, v in enumerate(row):
            c.level_scale[l][ch] = float(v)
    for l, v in enumerate(spec.level_tokens):
        c.level_tokens[l] = float(v)
    c.seed = int(spec.seed)
    for l, v in enumerate(spec.level_samples or []):
        c.level_samples[l] = int(v)
    c.n_families = int(spec.n_families or 0)
    for f in range(c.n_families):
        c.fam_len[f] = int(spec.fam_len[f])
        c.fam_channels[f] = int(spec.fam_channels[f])
        c.fam_budget_q[f] = int(spec.fam_budget_q[f])
    return c


def net_desc(net: W.NetSpec) -> Net:
    return Net(net.obs_dim, net.hidden, net.n_actions, net.dtype)


def param_count(net: W.NetSpec) -> int:
    return int(lib().pe_param_count(C.byref(net_desc(net))))


class Env:
    """E environments over one trace (pe_env_create); the trace may be a
    host or device tensor."""

    def __init__(self, spec: W.EnvSpec, trace: torch.Tensor, phase: torch.Tensor):
        self.spec = spec
        self.cfg = env_config(spec)
        trace = trace.contiguous().to(torch.float32)
        phase = phase.contiguous().to(torch.uint8)
        h = C.c_void_p()
        _check(lib().pe_env_create(C.byref(self.cfg), _ptr(trace), _ptr(phase), C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().pe_env_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def state_bytes(self) -> int:
        return int(lib().pe_env_state_bytes(self._h))

    def save(self) -> bytes:
        buf = (C.c_uint8 * self.state_bytes())()
        _check(lib().pe_env_save(self._h, buf))
        return bytes(buf)

    def load(self, image: bytes):
        buf = (C.c_uint8 * len(image)).from_buffer_copy(image)
        _check(lib().pe_env_load(self._h, buf))


def alloc_rollout(spec: W.EnvSpec, net: W.NetSpec, T: int, device="cuda") -> Dict[str, torch.Tensor]:
    E, D = spec.n_envs, net.obs_dim
    odt = torch.float32 if net.dtype == PE_F32 else torch.bfloat16
    kw = dict(device=device)
    return dict(
        obs=torch.empty((T, E, D), dtype=odt, **kw), obs_last=torch.empty((E, D), dtype=odt, **kw),
        act=torch.empty((T, E), dtype=torch.uint8, **kw), logp=torch.empty((T, E), **kw),
        value=torch.empty((T, E), **kw), last_value=torch.empty(E, **kw),
        reward=torch.empty((T, E), **kw), done=torch.empty((T, E), dtype=torch.uint8, **kw),
        viol=torch.empty((E, 2), dtype=torch.int32, **kw), tokens=torch.empty(E, **kw),
        excess=torch.empty(E, **kw), energy_q=torch.empty(E, dtype=torch.int64, **kw),
        samples=torch.empty(E, dtype=torch.int64, **kw), q=torch.empty((T, E), dtype=torch.int32, **kw))


def _rollout_buf(b: Dict[str, Optional[torch.Tensor]]) -> RolloutBuf:
    return RolloutBuf(*[(b[k].data_ptr() if b.get(k) is not None else None) for k in ROLLOUT_FIELDS])


def rollout_workspace_bytes(env: Env, net: W.NetSpec) -> int:
    return int(lib().pe_rollout_workspace_bytes(env._h, C.byref(net_desc(net))))


def alloc_workspace(nbytes: int, device="cuda") -> Optional[torch.Tensor]:
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def rollout(env: Env, net: W.NetSpec, params: torch.Tensor, T: int, iteration: int,
            buf: Dict[str, torch.Tensor], lam: float = 1.0, deterministic: bool = False,
            workspace: Optional[torch.Tensor] = None, stream=None):
    rb = _rollout_buf(buf)
    if workspace is None and net.dtype != PE_F32:
        workspace = alloc_workspace(rollout_workspace_bytes(env, net))
    nbytes = 0 if workspace is None else workspace.numel()
    _check(lib().pe_rollout(env._h, C.byref(net_desc(net)), _ptr(params), T, iteration, lam,
                            PE_ROLLOUT_DETERMINISTIC if deterministic else 0, C.byref(rb),
                            _ptr(workspace), nbytes, _stream(stream)))


def set_offsets(env: Env, offsets: torch.Tensor, stream=None):
    """Start a new episode of every env at offsets[e] (int32 device tensor)."""
    _check(lib().pe_env_set_offsets(env._h, _ptr(offsets), _stream(stream)))


def alloc_rule_rollout(spec: W.EnvSpec, T: int, obs: bool = False, obs_bf16: bool = False,
                       device="cuda") -> Dict[str, torch.Tensor]:
    """Buffers of a rule-policy rollout (observations only if asked for)."""
    E, D = spec.n_envs, spec.obs_dim
    kw = dict(device=device)
    odt = torch.bfloat16 if obs_bf16 else torch.float32
    return dict(
        obs=torch.empty((T, E, D), dtype=odt, **kw) if obs else None,
        obs_last=torch.empty((E, D), dtype=odt, **kw) if obs else None,
        act=torch.empty((T, E), dtype=torch.uint8, **kw), logp=None, value=None, last_value=None,
        reward=torch.empty((T, E), **kw), done=torch.empty((T, E), dtype=torch.uint8, **kw),
        viol=torch.empty((E, 2), dtype=torch.int32, **kw), tokens=torch.empty(E, **kw),
        excess=torch.empty(E, **kw), energy_q=torch.empty(E, dtype=torch.int64, **kw),
        samples=torch.empty(E, dtype=torch.int64, **kw), q=torch.empty((T, E), dtype=torch.int32, **kw))


def rollout_rule(env: Env, rule: W.RuleSpec, T: int, iteration: int, buf: Dict[str, torch.Tensor],
                 lam: float = 1.0, stream=None):
    """T steps of every env under a baseline rule policy (no network)."""
    rb = _rollout_buf(buf)
    obs_bf16 = buf["obs"] is not None and buf["obs"].dtype == torch.bfloat16
    r = Rule(rule.kind, rule.hi_q, rule.lo_q, rule.drop30_q, rule.climb30_q, rule.climb10_q)
    _check(lib().pe_rollout_rule(env._h, C.byref(r), T, iteration, lam, int(obs_bf16), C.byref(rb),
                                 _stream(stream)))


def rollout_replay(env: Env, actions: torch.Tensor, T: int, iteration: int, buf: Dict[str, torch.Tensor],
                   lam: float = 1.0, stream=None):
    """Teacher-forced rollout: env e takes actions[t][e] (uint8, device, [T][E]) at step t."""
    if actions.dtype != torch.uint8 or actions.numel() != T * env.spec.n_envs or not actions.is_contiguous():
        raise ValueError("actions must be a contiguous uint8 tensor of T x n_envs")
    rb = _rollout_buf(buf)
    obs_bf16 = buf["obs"] is not None and buf["obs"].dtype == torch.bfloat16
    _check(lib().pe_rollout_replay(env._h, _ptr(actions), T, iteration, lam, int(obs_bf16), C.byref(rb),
                                   _stream(stream)))


def wait_selftest(mode: int, limit_cycles: int, workspace: torch.Tensor, stream=None):
    """Run one of the library's bounded waits with a short budget (see pe.h);
    raises PEError with PE_ETIMEOUT when the wait gives up."""
    if workspace.numel() * workspace.element_size() < (1 << 26 if mode in (3, 4) else 16):
        raise ValueError("workspace too small")
    _check(lib().pe_wait_selftest(mode, int(limit_cycles), _ptr(workspace), _stream(stream)))


def dual_ascent(viol: torch.Tensor, steps: int, lam: torch.Tensor, rate: Optional[torch.Tensor] = None,
                target: float = 0.08, eta: float = 0.5, lo: float = 1e-3, hi: float = 2.0, window: int = 60,
                additive: bool = False, stream=None):
    """Eq. 7 update of the device scalar lam (float32) from a rollout's viol counts."""
    _check(lib().pe_dual_ascent(_ptr(viol), viol.shape[0], steps, window, int(additive), target, eta, lo, hi,
                                _ptr(lam), _ptr(rate), _stream(stream)))


def value_workspace_bytes(net: W.NetSpec) -> int:
    return int(lib().pe_value_workspace_bytes(C.byref(net_desc(net))))


def value(net: W.NetSpec, params: torch.Tensor, obs: torch.Tensor, out: torch.Tensor,
          workspace: Optional[torch.Tensor] = None, stream=None):
    n = obs.numel() // net.obs_dim
    if workspace is None and net.dtype != PE_F32:
        workspace = alloc_workspace(value_workspace_bytes(net))
    nbytes = 0 if workspace is None else workspace.numel()
    _check(lib().pe_value(C.byref(net_desc(net)), _ptr(params), _ptr(obs), n, _ptr(out),
                          _ptr(workspace), nbytes, _stream(stream)))


def device_check(stream=None):
    """Synchronise and raise PEError(PE_ETIMEOUT) if a bounded device wait gave up."""
    _check(lib().pe_device_check(_stream(stream)))


def gae(reward, value_, done, last_value, gamma: float, lam: float, adv, ret, stream=None):
    T, E = reward.shape
    _check(lib().pe_gae(_ptr(reward), _ptr(value_), _ptr(done), _ptr(last_value), T, E, gamma,
                        lam, _ptr(adv), _ptr(ret), _stream(stream)))


def ppo_config(ppo: W.PPOSpec, seed: int, iteration: int) -> PPOConfig:
    c = PPOConfig()
    c.epochs, c.minibatch = ppo.epochs, ppo.minibatch
    for n in ("lr", "clip", "vf_coef", "ent_coef", "max_grad_norm", "beta1", "beta2", "eps"):
        setattr(c, n, float(getattr(ppo, n)))
    c.seed, c.iteration = seed, iteration
    return c


def ppo_workspace_bytes(net: W.NetSpec, ppo: W.PPOSpec, n: int) -> int:
    c = ppo_config(ppo, 0, 0)
    return int(lib().pe_ppo_workspace_bytes(C.byref(net_desc(net)), C.byref(c), n))


def ppo_update(net: W.NetSpec, ppo: W.PPOSpec, params, adam_m, adam_v, adam_t: int, obs, act,
               logp_old, adv, ret, stats, workspace, seed: int, iteration: int, stream=None):
    c = ppo_config(ppo, seed, iteration)
    n = act.numel()
    _check(lib().pe_ppo_update(C.byref(net_desc(net)), _ptr(params), _ptr(adam_m), _ptr(adam_v),
                               adam_t, _ptr(obs), _ptr(act), _ptr(logp_old), _ptr(adv), _ptr(ret),
                               n, C.byref(c), _ptr(stats), _ptr(workspace), workspace.numel(),
                               _stream(stream)))


def fleet_workspace_bytes(J: int, L: int, H: int) -> int:
    return int(lib().pe_fleet_workspace_bytes(J, L, H))


def fleet_windows(traces, job_of_gpu, J: int, offsets, H: int, windows: Sequence[int],
                  budget_q: int, counts, peaks, workspace, stream=None):
    G, L = traces.shape
    N = offsets.shape[0]
    w = (C.c_int32 * len(windows))(*[int(x) for x in windows])
    _check(lib().pe_fleet_windows(_ptr(traces), G, L, _ptr(job_of_gpu), J, _ptr(offsets), N, H,
                                  w, len(windows), budget_q, _ptr(counts), _ptr(peaks),
                                  _ptr(workspace), workspace.numel(), _stream(stream)))


def fleet_stagger_workspace_bytes(J: int, L: int, H: int, stride: int) -> int:
    return int(lib().pe_fleet_stagger_workspace_bytes(J, L, H, stride))


def fleet_stagger(traces, job_of_gpu, J: int, H: int, w: int, stride: int, offsets, peaks, workspace,
                  stream=None):
    """Greedy phase-staggered start offsets (offsets[J]) and stage peaks (peaks[J])."""
    G, L = traces.shape
    _check(lib().pe_fleet_stagger(_ptr(traces), G, L, _ptr(job_of_gpu), J, H, w, stride, _ptr(offsets),
                                  _ptr(peaks), _ptr(workspace), workspace.numel(), _stream(stream)))


PE_ROOF_FFMA, PE_ROOF_FFMA2, PE_ROOF_IADD, PE_ROOF_L2 = 0, 1, 2, 3


def roof_probe(kind: int, buf, reps: int, stream=None):
    """(device ms, units) of one timed throughput loop (pe_roof_probe)."""
    ms, units = C.c_double(0.0), C.c_double(0.0)
    _check(lib().pe_roof_probe(kind, _ptr(buf), buf.numel() * buf.element_size(), reps, C.byref(ms),
                               C.byref(units), _stream(stream)))
    return ms.value, units.value


FLEET_NOALLOC_SCRATCH_BYTES = 4 * 1024 * 1024


def fleet_windows_noalloc(traces, job_of_gpu, J: int, offsets, H: int, windows: Sequence[int],
                          budget_q: int, counts, peaks, stream=None):
    """pe_fleet_windows without a workspace, for callers that cannot allocate
    device memory; its scratch is a fixed 4 MiB array inside the library."""
    G, L = traces.shape
    N = offsets.shape[0]
    w = (C.c_int32 * len(windows))(*[int(x) for x in windows])
    _check(lib().pe_fleet_windows_noalloc(_ptr(traces), G, L, _ptr(job_of_gpu), J, _ptr(offsets), N,
                                          H, w, len(windows), budget_q, _ptr(counts), _ptr(peaks),
                                          _stream(stream)))


# ---------------------------------------------------------------------------
# token operators: generation over a paged cache, and scoring with its gradient
# ---------------------------------------------------------------------------
_DTYPE = {torch.float32: PE_F32, torch.bfloat16: PE_BF16, torch.float16: PE_F16}


_current_device = torch._C._cuda_getDevice
_INT32 = 2 ** 31 - 1  # the largest size of an int32 argument; ctypes drops what is above


def _stream_of(dev: int, stream=None) -> int:
    """The given stream, or the device's current one (by its handle alone:
    building a Stream object costs more than the launch)."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev)


def _launch_device(name: str, t: torch.Tensor) -> int:
    """Device of a call: that of its tensors, which has to be the current one,
    where the library launches."""
    dev = t.get_device()
    if dev < 0 or dev != _current_device():
        raise ValueError(f"{name} must be on the current CUDA device")
    return dev


def _want(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _vec(name: str, t: torch.Tensor, n: int, dtype: torch.dtype, dev: int) -> int:
    """Device pointer of a contiguous vector of n elements."""
    if t.dtype is not dtype or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on device {dev}")
    return t.data_ptr()


def _heads(name: str, t: torch.Tensor, shape: tuple, dtype: torch.dtype, dev: int):
    """(pointer, row stride, head stride) of an [n][heads][head_dim] tensor."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev:
        s0, s1, s2 = t.stride()
        if s2 == 1:
            return t.data_ptr(), s0 if shape[0] > 1 else 0, s1 if shape[1] > 1 else 0
    raise ValueError(f"{name} must be a {dtype} tensor of {list(shape)} on device {dev} with adjacent elements")


class KVCache:
    """A paged cache of keys and values (pe_kv_cache): k and v are
    [pages, slots, heads, head_dim] tensors of bf16, fp16 or float8_e4m3fn with
    equal strides (a transposed view of [pages, heads, slots, head_dim] storage
    will do), table is [sequences, pages of a sequence] int32.  A cache of
    float8_e4m3fn has scales (pe_kv_scales): k_scale and v_scale are
    [pages, slots, heads] tensors of uint8 or float8_e8m0fnu with equal strides.
    Holds the tensors; the table's entries may change between calls.  The calls
    below run on the current device, where all of their tensors have to be."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        _want(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype
              and k.dtype in (torch.bfloat16, torch.float16, torch.float8_e4m3fn) and k.is_cuda and v.is_cuda and k.stride(3) == 1,
              "k and v must be bf16, fp16 or float8_e4m3fn device tensors of [pages, slots, heads, head_dim] with equal "
              "strides and adjacent elements")
        _want(table.dim() == 2 and table.dtype == torch.int32 and table.is_cuda and (table.shape[1] < 2 or table.stride(1) == 1),
              "table must be an int32 device tensor of [sequences, pages] with adjacent entries")
        _want(max(table.shape) <= _INT32 and max(k.shape[1:]) <= _INT32, "sizes must be below 2^31")
        _want(table.shape[0] < 2 or table.stride(0) >= table.shape[1], "table's rows must not overlap (an expanded row is no table)")
        _want(k.get_device() == v.get_device() == table.get_device(), "k, v and table must be on one device")
        self.k, self.v, self.table, self.k_scale, self.v_scale = k, v, table, k_scale, v_scale
        st = [k.stride(i) if k.shape[i] > 1 else 0 for i in range(3)]
        self.n_seqs, self.n_heads, self.head_dim, self.page_size = table.shape[0], k.shape[2], k.shape[3], k.shape[1]
        self.eight = k.dtype == torch.float8_e4m3fn
        self.dtype = k.dtype
        self._desc = KVCacheDesc(k.data_ptr(), v.data_ptr(), table.data_ptr(), k.shape[0], st[0], st[1], st[2],
                                 table.stride(0) if table.shape[0] > 1 else table.shape[1], table.shape[0], table.shape[1], k.shape[1],
                                 k.shape[2], k.shape[3], PE_E4M3 if self.eight else _DTYPE[k.dtype])
        self._ref = C.byref(self._desc)
        self._scales = None
        if not self.eight:
            _want(k_scale is None and v_scale is None, "a 16-bit cache has no scales")
            return
        _want(k_scale is not None and v_scale is not None and k_scale.shape == v_scale.shape == k.shape[:3]
              and k_scale.stride() == v_scale.stride() and k_scale.dtype == v_scale.dtype
              and k_scale.dtype in (torch.uint8, torch.float8_e8m0fnu)
              and k_scale.get_device() == v_scale.get_device() == k.get_device(),
              "an 8-bit cache needs k_scale and v_scale, uint8 or float8_e8m0fnu device tensors of [pages, slots, heads] "
              "with equal strides")
        ss = [k_scale.stride(i) if k.shape[i] > 1 else 0 for i in range(3)]
        _want(all(x > 0 for x, n in zip(ss, k.shape) if n > 1), "rows of an 8-bit cache must not share a scale")
        self._scale_desc = KVScales(k_scale.data_ptr(), v_scale.data_ptr(), *ss)
        self._scales = C.byref(self._scale_desc)

    def _type(self, name: str, t: torch.Tensor) -> torch.dtype:
        """dtype of what goes in or comes out: the cache's, or t's where that has 8 bits."""
        if not self.eight:
            return self.dtype
        _want(t.dtype in (torch.bfloat16, torch.float16), f"{name} must be bf16 or fp16")
        return t.dtype


def rot_table(max_pos: int, rot_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """Rotation table of kv_append: row p holds cos(p f_i), then sin(p f_i),
    with f_i = base^(-2 i / rot_dim), evaluated in fp64 and rounded to fp32."""
    f = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    ang = torch.arange(max_pos, dtype=torch.float64)[:, None] * f
    return torch.cat([torch.cos(ang), torch.sin(ang)], 1).float().to(device)


def kv_append(cache: KVCache, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor,
              seqs: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
              q_out: Optional[torch.Tensor] = None, rot: Optional[torch.Tensor] = None, interleaved: bool = False,
              stream=None, slots: Optional[torch.Tensor] = None):
    """Append keys and values of new tokens ([tokens, heads, head_dim]) at
    their positions (int32), rotating q (into q_out, default in place) and k
    by position with rot ([positions, rot_dim], see rot_table); token t is of
    sequence seqs[t], or t where seqs is None.  With slots (int32) token t is
    written to position slots[t] and not where its rotation says.  An 8-bit
    cache gets codes and scales of the rows (bf16 or fp16, like q)."""
    n, D, dt, dev = positions.numel(), cache.head_dim, cache._type("k", k), _launch_device("the cache", cache.k)
    kp, ks, kh = _heads("k", k, (n, cache.n_heads, D), dt, dev)
    vp, vs, vh = _heads("v", v, (n, cache.n_heads, D), dt, dev)
    qp = qs = qh = op = os_ = oh = hq = rp = max_pos = rot_dim = 0
    if q is not None:
        hq = q.shape[1]
        qp, qs, qh = _heads("q", q, (n, hq, D), dt, dev)
        op, os_, oh = (qp, qs, qh) if q_out is None else _heads("q_out", q_out, (n, hq, D), dt, dev)
    if rot is not None:
        if rot.dim() != 2 or rot.dtype is not torch.float32 or rot.get_device() != dev or not rot.is_contiguous():
            raise ValueError(f"rot must be a contiguous float32 tensor of [positions, rot_dim] on device {dev}")
        rp = rot.data_ptr()
        max_pos, rot_dim = rot.shape
    t = _KV_TOKENS(_vec("positions", positions, n, torch.int32, dev),
                   0 if seqs is None else _vec("seqs", seqs, n, torch.int32, dev), rp, qp, op, kp, vp, n, max_pos,
                   qs, qh, os_, oh, ks, kh, vs, vh, hq, rot_dim, interleaved)
    if cache.eight or slots is not None:
        at = None if slots is None else _vec("slots", slots, n, torch.int32, dev)
        _check(lib().pe_kv_append_at(cache._ref, cache._scales, t, at, _DTYPE[dt], _stream_of(dev, stream)))
    else:
        _check(lib().pe_kv_append(cache._ref, t, _stream_of(dev, stream)))


def decode_attn_workspace_bytes(cache: KVCache, n_q_heads: int) -> int:
    if cache.eight:
        return int(lib().pe_decode_attn8_workspace_bytes(cache._ref, n_q_heads))
    return int(lib().pe_decode_attn_workspace_bytes(cache._ref, n_q_heads))


def _workspace(workspace: Optional[torch.Tensor], nbytes, dev: int, stream) -> torch.Tensor:
    """The caller's workspace, or one of nbytes() bytes."""
    if workspace is None:
        with torch.cuda.stream(stream):  # of the stream that uses it (None: the current one)
            return alloc_workspace(nbytes())
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous, on device {dev}")
    return workspace


def decode_attn(cache: KVCache, q: torch.Tensor, lens: torch.Tensor, out: torch.Tensor, scale: Optional[float] = None,
                window: int = 0, lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream=None):
    """out[b] = attention of q[b] ([sequences, query heads, head_dim]) over the
    lens[b] (int32) positions of sequence b; scale defaults to head_dim^-1/2.
    q and out are of the cache's dtype, of bf16 or fp16 over an 8-bit cache."""
    n, hq, dev, dt = cache.n_seqs, q.shape[1], _launch_device("the cache", cache.k), cache._type("q", q)
    shape = (n, hq, cache.head_dim)
    qp, qs, qh = _heads("q", q, shape, dt, dev)
    op, os_, oh = _heads("out", out, shape, dt, dev)
    lp = _vec("lens", lens, n, torch.int32, dev)
    sp = None if lse is None else _vec("lse", lse, n * hq, torch.float32, dev)
    if abs(window) > _INT32:
        raise ValueError("window must be in [0, 2^31)")
    workspace = _workspace(workspace, lambda: decode_attn_workspace_bytes(cache, hq), dev, stream)
    scale = cache.head_dim ** -0.5 if scale is None else scale
    if cache.eight:
        _check(lib().pe_decode_attn8(cache._ref, cache._scales, _DTYPE[dt], qp, qs, qh, hq, lp, scale, window, op, os_, oh, sp,
                                     workspace.data_ptr(), workspace.numel(), _stream_of(dev, stream)))
    else:
        _check(lib().pe_decode_attn(cache._ref, qp, qs, qh, hq, lp, scale, window, op, os_, oh, sp, workspace.data_ptr(),
                                    workspace.numel(), _stream_of(dev, stream)))


def tree_attn_workspace_bytes(cache: KVCache, n_nodes: int, n_q_heads: int) -> int:
    return int(lib().pe_tree_attn_workspace_bytes(cache._ref, n_nodes, n_q_heads))


def _nodes(name: str, t: torch.Tensor, shape: tuple, dtype: torch.dtype, dev: int):
    """(pointer, sequence, node and head strides) of an [n][nodes][heads][head_dim] tensor."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev:
        s0, s1, s2, s3 = t.stride()
        if s3 == 1:
            return t.data_ptr(), s0 if shape[0] > 1 else 0, s1 if shape[1] > 1 else 0, s2 if shape[2] > 1 else 0
    raise ValueError(f"{name} must be a {dtype} tensor of {list(shape)} on device {dev} with adjacent elements")


def tree_attn(cache: KVCache, q: torch.Tensor, lens: torch.Tensor, mask: torch.Tensor, out: torch.Tensor,
              scale: Optional[float] = None, window: int = 0, lse: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of drafted tokens q ([sequences, nodes, query heads, head_dim],
    64 nodes at most): node i of sequence b, appended at position lens[b] + i,
    attends to the lens[b] positions ahead of the tree and to the nodes whose
    bits are set in mask[b, i] (int64 [sequences, nodes]; 0: padding).  A mask
    expanded from one row is a tree for all.  scale defaults to head_dim^-1/2."""
    dev = _launch_device("the cache", cache.k)
    _want(q.dim() == 4, "q must have the dimensions [sequences, nodes, query heads, head_dim]")
    n, nodes, hq, dt = cache.n_seqs, q.shape[1], q.shape[2], cache._type("q", q)
    shape = (n, nodes, hq, cache.head_dim)
    qp, qs, qn, qh = _nodes("q", q, shape, dt, dev)
    op, os_, on, oh = _nodes("out", out, shape, dt, dev)
    _want(mask.shape == (n, nodes) and mask.dtype is torch.int64 and mask.get_device() == dev
          and (nodes < 2 or mask.stride(1) == 1), f"mask must be an int64 tensor of {[n, nodes]} on device {dev} with adjacent entries")
    _want(nodes <= 64, "a tree has 64 nodes at most")
    if abs(window) > _INT32:
        raise ValueError("window must be in [0, 2^31)")
    sp = 0 if lse is None else _vec("lse", lse, n * nodes * hq, torch.float32, dev)
    t = _TREE_QUERIES(qp, op, sp, _vec("lens", lens, n, torch.int32, dev), mask.data_ptr(), qs, qn, qh, os_, on, oh,
                      mask.stride(0) if n > 1 else 0, nodes, hq, _DTYPE[dt])
    workspace = _workspace(workspace, lambda: tree_attn_workspace_bytes(cache, nodes, hq), dev, stream)
    _check(lib().pe_tree_attn(cache._ref, cache._scales, t, cache.head_dim ** -0.5 if scale is None else scale, window,
                              workspace.data_ptr(), workspace.numel(), _stream_of(dev, stream)))


def _moves(name: str, t: torch.Tensor, shape, dev: int):
    if t.shape == shape and t.dtype is torch.int32 and t.get_device() == dev and (shape[1] < 2 or t.stride(1) == 1):
        return t.data_ptr(), t.stride(0) if shape[0] > 1 else shape[1]
    raise ValueError(f"{name} must be an int32 tensor of {list(shape)} on device {dev} with adjacent entries")


def kv_move(cache: KVCache, src: torch.Tensor, dst: torch.Tensor, stream=None):
    """Position dst[b, i] of sequence b gets what position src[b, i] held before
    the call (int32 [sequences, moves], 64 moves at most; out of range: no move)."""
    dev = _launch_device("the cache", cache.k)
    _want(src.dim() == 2 and src.shape[0] == cache.n_seqs and src.shape[1] <= 64, "src must be [sequences, moves], 64 moves at most")
    shape = src.shape
    sp, ss = _moves("src", src, shape, dev)
    dp, ds = _moves("dst", dst, shape, dev)
    _check(lib().pe_kv_move(cache._ref, cache._scales, sp, ss, dp, ds, shape[1], _stream_of(dev, stream)))


def _rows(name: str, t: torch.Tensor, dev: int):
    """(pointer, dtype, rows, columns, row stride) of a matrix of logits."""
    dt = _DTYPE.get(t.dtype)
    if dt is not None and t.get_device() == dev and t.ndim == 2:
        (n, V), (rs, cs) = t.shape, t.stride()
        if (cs == 1 or V < 2) and V <= _INT32:
            return t.data_ptr(), dt, n, V, rs if n > 1 else V
    raise ValueError(f"{name} must be a float32, bf16 or fp16 tensor of [rows, V] on device {dev} with adjacent elements")


def token_logp(logits: torch.Tensor, tokens: Optional[torch.Tensor], logp: Optional[torch.Tensor],
               entropy: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               top_logp: Optional[torch.Tensor] = None, top_id: Optional[torch.Tensor] = None, scale: float = 1.0,
               stream=None):
    """Log-probabilities (fp32) of tokens (int32, negative: no target) under
    softmax(scale * logits), with the rows' entropies, log sums and top
    alternatives (top_logp fp32 and top_id int32, [rows, k]) where asked for."""
    dev = _launch_device("logits", logits)
    p, dt, n, V, rs = _rows("logits", logits, dev)
    f = torch.float32
    k = 0
    if top_id is not None or top_logp is not None:
        _want(top_id is not None and top_logp is not None and top_id.dim() == 2, "top_logp and top_id go together, [rows, k]")
        k = top_id.shape[1]
    _check(lib().pe_token_logp(
        p, dt, n, V, rs, None if tokens is None else _vec("tokens", tokens, n, torch.int32, dev), scale,
        None if logp is None else _vec("logp", logp, n, f, dev), None if entropy is None else _vec("entropy", entropy, n, f, dev),
        None if lse is None else _vec("lse", lse, n, f, dev), k, None if not k else _vec("top_logp", top_logp, n * k, f, dev),
        None if not k else _vec("top_id", top_id, n * k, torch.int32, dev), _stream_of(dev, stream)))


def token_logp_grad(logits: torch.Tensor, tokens: Optional[torch.Tensor], lse: torch.Tensor, dlogits: torch.Tensor,
                    g_logp: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                    g_entropy: Optional[torch.Tensor] = None, scale: float = 1.0, stream=None):
    """dlogits = gradient of sum(g_logp logp) + sum(g_entropy entropy) in the
    logits, from token_logp's lse and entropy; dlogits may be logits itself."""
    dev = _launch_device("logits", logits)
    p, dt, n, V, rs = _rows("logits", logits, dev)
    dp, ddt, dn, dV, ds = _rows("dlogits", dlogits, dev)
    _want(ddt == dt and dn == n and dV == V, "dlogits must have the logits' shape and dtype")
    f = torch.float32
    _check(lib().pe_token_logp_grad(
        p, dt, n, V, rs, None if tokens is None else _vec("tokens", tokens, n, torch.int32, dev), scale,
        _vec("lse", lse, n, f, dev), None if entropy is None else _vec("entropy", entropy, n, f, dev),
        None if g_logp is None else _vec("g_logp", g_logp, n, f, dev),
        None if g_entropy is None else _vec("g_entropy", g_entropy, n, f, dev), dp, ds, _stream_of(dev, stream)))


def profile_enable(on: bool):
    _check(lib().pe_profile_enable(int(bool(on))))


def profile_read(kind: int):
    """(summed device ms, launches) of one kernel kind since the last read."""
    ms = C.c_double()
    n = C.c_int64()
    _check(lib().pe_profile_read(kind, C.byref(ms), C.byref(n)))
    return ms.value, n.value


def profile_kind_name(kind: int) -> str:
    return lib().pe_profile_kind_name(kind).decode()
