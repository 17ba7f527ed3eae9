"""Python binding of libwam with the same entry points as the C ABI.

PyTorch only provides device memory and the HIP stream; every step of the
denoising path and of the adaptation operators runs in libwam's kernels.
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from array import array
from dataclasses import dataclass
from typing import NamedTuple

import numpy as np
import torch

from . import _lib as abi


class WamError(RuntimeError):
    pass


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        if not t.is_cuda:
            raise WamError("libwam takes device tensors only")
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise WamError("device tensors must be contiguous float32")
        return C.c_void_p(t.data_ptr())
    return C.c_void_p(int(t))


def host_weight_order(n_layers: int) -> list[str]:
    """Names of the canonical host weight buffer, in the order wam.h documents."""
    names = ["t_w1", "t_b1", "t_w2", "t_b2", "in_wv", "in_bv", "in_wa", "in_ba", "in_wo", "in_bo"]
    for l in range(n_layers):
        names += [f"l{l}.{n}" for n in ("mod_w", "mod_b", "qkv_w", "qkv_b", "q_g", "k_g", "proj_w",
                                        "proj_b", "fc1_w", "fc1_b", "fc2_w", "fc2_b")]
    names += ["f_mod_w", "f_mod_b", "out_wv", "out_bv", "out_wa", "out_ba"]
    return names


def make_config(B, L, D, H, F, Nv, Cv, Na, A, No, Co, dtype="bf16", qk_norm=True, ln_eps=1e-6) -> abi.WamConfig:
    return abi.WamConfig(B=B, L=L, D=D, H=H, F=F, Nv=Nv, Cv=Cv, Na=Na, A=A, No=No, Co=Co,
                       dtype={"bf16": abi.WAM_BF16, "fp8": abi.WAM_FP8}.get(dtype, abi.WAM_FP32), qk_norm=int(bool(qk_norm)),
                       ln_eps=ln_eps)


def config_of(spec) -> abi.WamConfig:
    """Config from any object exposing the model fields (B, L, D, ...)."""
    return make_config(spec.B, spec.L, spec.D, spec.H, spec.F, spec.Nv, spec.Cv, spec.Na, spec.A,
                       spec.No, spec.Co, spec.dtype, spec.qk_norm, spec.ln_eps)


def rr_profile(q=0, s=0, e=0, mode=abi.WAM_RR_OFF, alpha_min=1.0, alpha_max=1.25, eps=1e-8,
               gamma_cos=0.80, gamma_fit=0.60, branches=abi.WAM_RR_JOINT) -> abi.WamRRProfile:
    return abi.WamRRProfile(q=q, s=s, e=e, mode=mode, alpha_min=alpha_min, alpha_max=alpha_max, eps=eps,
                          gamma_cos=gamma_cos, gamma_fit=gamma_fit, branches=branches)


@dataclass
class StepInfo:
    rr_active: bool
    attempted: bool
    accepted: bool
    layers_evaluated: int
    layers_skipped: int
    alpha: np.ndarray
    cos: np.ndarray
    fit: np.ndarray

    @classmethod
    def of(cls, s: abi.WamStepInfo, B: int) -> "StepInfo":
        a = np.array([[s.alpha[b][i] for i in range(2)] for b in range(B)])
        c = np.array([[s.cos[b][i] for i in range(2)] for b in range(B)])
        f = np.array([[s.fit[b][i] for i in range(2)] for b in range(B)])
        return cls(bool(s.rr_active), bool(s.rr_attempted), bool(s.rr_accepted), s.layers_evaluated,
                   s.layers_skipped, a, c, f)


class WamModel:
    """One libwam handle with its device weights and workspace (torch-owned)."""

    def __init__(self, cfg: abi.WamConfig, weights: dict, device="cuda", stream: torch.cuda.Stream | None = None,
                 own_stream: bool = False):
        if not torch.cuda.is_available():
            raise WamError("libwam needs a HIP device")
        self.lib = abi.lib()
        self.cfg = cfg
        self.device = torch.device(device)
        self.B = cfg.B
        self.traj = int(self.lib.wam_traj_elems(C.byref(cfg)))
        n_host = int(self.lib.wam_host_weight_count(C.byref(cfg)))
        wbytes = int(self.lib.wam_weight_bytes(C.byref(cfg)))
        wsbytes = int(self.lib.wam_workspace_bytes(C.byref(cfg)))
        if n_host == 0 or wbytes == 0:
            raise WamError("invalid configuration")
        host = np.concatenate([np.ascontiguousarray(weights[n], np.float32).ravel()
                               for n in host_weight_order(cfg.L)])
        if host.size != n_host:
            raise WamError(f"weight count {host.size} != {n_host}")
        if own_stream:  # a dedicated (default-priority) stream, required for graph replay
            stream = torch.cuda.Stream(self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.wdev = torch.empty(wbytes, dtype=torch.uint8, device=self.device)
        self.ws = torch.empty(wsbytes, dtype=torch.uint8, device=self.device)
        h = C.c_void_p()
        st = self.lib.wam_init(C.byref(cfg), host.ctypes.data_as(C.c_void_p), host.size,
                               C.c_void_p(self.wdev.data_ptr()), wbytes, C.c_void_p(self.ws.data_ptr()),
                               wsbytes, C.c_void_p(self.stream.cuda_stream), C.byref(h))
        if st != abi.WAM_OK:
            raise WamError(f"wam_init failed: {self.lib.wam_status_string(st).decode()}")
        self.h = h
        self.K = 0

    # ------------------------------------------------------------ helpers
    def _enter(self):
        """Order the handle's stream after torch's current stream (inputs)."""
        cur = torch.cuda.current_stream(self.device)
        if cur.cuda_stream != self.stream.cuda_stream:
            self.stream.wait_stream(cur)

    def _leave(self):
        """Order torch's current stream after the handle's stream (outputs)."""
        cur = torch.cuda.current_stream(self.device)
        if cur.cuda_stream != self.stream.cuda_stream:
            cur.wait_stream(self.stream)

    def _check(self, st, what):
        if st != abi.WAM_OK:
            msg = self.lib.wam_last_error(self.h).decode()
            raise WamError(f"{what}: {self.lib.wam_status_string(st).decode()}: {msg}")

    def close(self):
        if getattr(self, "h", None):
            self.lib.wam_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def new_traj(self):
        return torch.empty((self.B, self.traj), dtype=torch.float32, device=self.device)

    # ------------------------------------------------------------ ABI
    def set_schedule(self, sigmas):
        s = np.ascontiguousarray(sigmas, np.float32)
        self._check(self.lib.wam_set_schedule(self.h, s.ctypes.data_as(C.POINTER(C.c_float)), s.size - 1),
                    "wam_set_schedule")
        self.K = s.size - 1

    def set_rotary(self, pos, sections=None, freq=None, layout="halves", keep_table=False):
        """Rotary positions of the rows (wam_set_rotary): pos float32 [T, 3] on the
        device, one frequency per pair; pos None: back to the additive table alone."""
        if pos is None:
            self._check(self.lib.wam_set_rotary(self.h, None), "wam_set_rotary")
            self._pos = None
            return
        if not isinstance(pos, torch.Tensor) or sections is None or freq is None:
            raise WamError("set_rotary: needs positions, sections and frequencies")
        T = self.cfg.Nv + self.cfg.Na + self.cfg.No
        if tuple(pos.shape) != (T, 3):
            raise WamError(f"set_rotary: pos must be [{T}, 3]")
        ladder = np.ascontiguousarray(freq, np.float64)
        if len(sections) != 3 or ladder.shape != (sum(sections),):
            raise WamError("set_rotary: needs three sections and one frequency per pair")
        self._enter()
        a = abi.WamRotaryArgs(pos=_ptr(pos), sections=(C.c_int32 * 3)(*sections),
                              layout=_choice(_LAYOUTS, layout, "set_rotary: layout"), freq=ladder.ctypes.data,
                              keep_table=int(bool(keep_table)))
        self._check(self.lib.wam_set_rotary(self.h, C.byref(a)), "wam_set_rotary")
        self._pos = pos  # read by every step

    def set_post_norm(self, gains):
        """RMS post-norms of both blocks of every layer (wam_set_post_norm): gains
        float32 [L, 2, D] on the device, or None."""
        if gains is not None and tuple(gains.shape) != (self.cfg.L, 2, self.cfg.D):
            raise WamError(f"set_post_norm: gains must be {(self.cfg.L, 2, self.cfg.D)}")
        self._enter()
        self._check(self.lib.wam_set_post_norm(self.h, _ptr(gains)), "wam_set_post_norm")
        self._gains = gains  # read by every step

    def velocity(self, k, x, cond, v_out=None, rr=None):
        self._enter()
        v_out = self.new_traj() if v_out is None else v_out
        info = abi.WamStepInfo()
        self._check(self.lib.wam_velocity(self.h, k, _ptr(x), _ptr(cond), _ptr(v_out),
                                          C.byref(rr) if rr is not None else None, C.byref(info)),
                    "wam_velocity")
        self._leave()
        return v_out, StepInfo.of(info, self.B)

    def denoise_step(self, k, x, cond, rr=None):
        self._enter()
        info = abi.WamStepInfo()
        self._check(self.lib.wam_denoise_step(self.h, k, _ptr(x), _ptr(cond),
                                              C.byref(rr) if rr is not None else None, C.byref(info)),
                    "wam_denoise_step")
        self._leave()
        return StepInfo.of(info, self.B)

    def continue_(self, k_from, k_to, x, cond, rr=None, capture_stage=-1, x_capture=None):
        self._enter()
        n = max(k_to - k_from, 1)
        infos = (abi.WamStepInfo * n)()
        self._check(self.lib.wam_continue(self.h, k_from, k_to, _ptr(x), _ptr(cond),
                                          C.byref(rr) if rr is not None else None, capture_stage,
                                          _ptr(x_capture), infos), "wam_continue")
        self._leave()
        return [StepInfo.of(infos[i], self.B) for i in range(k_to - k_from)]

    def hidden(self, k, x, cond, n_layers, h_out=None):
        self._enter()
        if h_out is None:
            T = self.cfg.Nv + self.cfg.Na + self.cfg.No
            h_out = torch.empty((self.B, T, self.cfg.D), dtype=torch.float32, device=self.device)
        self._check(self.lib.wam_hidden(self.h, k, _ptr(x), _ptr(cond), n_layers, _ptr(h_out)), "wam_hidden")
        self._leave()
        return h_out

    def remap(self, x_bar, x_r, sigma_r, sigma_b0, shift_action, shift_video, noise, x_out=None):
        self._enter()
        x_out = self.new_traj() if x_out is None else x_out
        a = abi.WamRemapArgs(x_bar=_ptr(x_bar), x_r=_ptr(x_r), sigma_r=sigma_r, sigma_b0=sigma_b0,
                           shift_action=shift_action, shift_video=shift_video, noise=_ptr(noise), x_out=_ptr(x_out))
        self._check(self.lib.wam_adapt_state(self.h, abi.WAM_ADAPT_REMAP, C.byref(a)), "wam_adapt_state(REMAP)")
        self._leave()
        return x_out

    def rebind(self, cond):
        """Observation Rebinding's rebinding step (WAM_ADAPT_REBIND): the retained
        state continues under cond; cond=None in later step calls means it."""
        self._enter()
        a = abi.WamRebindArgs(cond=_ptr(cond))
        self._check(self.lib.wam_adapt_state(self.h, abi.WAM_ADAPT_REBIND, C.byref(a)), "wam_adapt_state(REBIND)")

    def reset_layer_state(self):
        self._check(self.lib.wam_adapt_state(self.h, abi.WAM_ADAPT_RESET_LAYER, None), "RESET_LAYER")

    def reset_all(self):
        self._check(self.lib.wam_adapt_state(self.h, abi.WAM_ADAPT_RESET_ALL, None), "RESET_ALL")

    def set_replan_state(self, x_bar, x_r, kappa):
        self._enter()
        a = abi.WamReplanStateArgs(x_bar=_ptr(x_bar), x_r=_ptr(x_r), kappa=kappa)
        self._check(self.lib.wam_adapt_state(self.h, abi.WAM_ADAPT_SET_REPLAN, C.byref(a)), "SET_REPLAN")

    def get_replan_state(self):
        self._enter()
        xb, xr = self.new_traj(), self.new_traj()
        kappa = C.c_int32()
        self._check(self.lib.wam_get_replan_state(self.h, _ptr(xb), _ptr(xr), C.byref(kappa)),
                    "wam_get_replan_state")
        self._leave()
        return xb, xr, kappa.value

    def consistency_score(self, u_hat, u, delta, weight):
        self._enter()
        n = len(u_hat)
        uh = (C.c_void_p * n)(*[_ptr(t).value for t in u_hat])
        uu = (C.c_void_p * n)(*[_ptr(t).value for t in u])
        cnt = (C.c_int64 * n)(*[t.numel() for t in u])
        dl = (C.c_double * n)(*delta)
        wt = (C.c_double * n)(*weight)
        S = C.c_double()
        self._check(self.lib.wam_consistency_score(self.h, n, uh, uu, cnt, dl, wt, C.byref(S)),
                    "wam_consistency_score")
        self._leave()
        return S.value

    def pack_condition(self, obs, n_obs, c_obs, ctx, n_ctx, c_ctx, ctx_stride, out):
        """out [B][No][Co] = obs tokens then ctx tokens, zero-padded (wam_pack_condition)."""
        self._enter()
        self._check(self.lib.wam_pack_condition(self.h, _ptr(obs), n_obs, c_obs, _ptr(ctx), n_ctx, c_ctx,
                                                ctx_stride, _ptr(out)), "wam_pack_condition")
        self._leave()
        return out

    def replan_args(self, cond_real, x_out, noise_remap, *, cond_pred=None, u_hat=(), u=(), delta=(), weight=(),
                    noise_first=None, rr=None, b0=0, r=0, shift_action=0, shift_video=0, k1=0, tau=0.5,
                    kappa_max=3, tr_enabled=True, or_enabled=True, rr_first=True, rr_prefix=True,
                    rr_refresh=True):
        """The wam_replan_args struct (device buffers referenced, not copied)."""
        a = abi.WamReplanArgs()
        a.cond_real = _ptr(cond_real)
        a.cond_pred = _ptr(cond_pred)
        a.n_components = len(u)
        for m in range(len(u)):
            a.u_hat[m] = _ptr(u_hat[m]).value
            a.u[m] = _ptr(u[m]).value
            a.n[m] = u[m].numel()
            a.delta[m] = delta[m]
            a.weight[m] = weight[m]
        a.noise_first = _ptr(noise_first)
        a.noise_remap = _ptr(noise_remap)
        a.x_out = _ptr(x_out)
        a.rr = rr if rr is not None else rr_profile()
        a.b0, a.r, a.shift_action, a.shift_video, a.k1 = b0, r, shift_action, shift_video, k1
        a.tau, a.kappa_max = tau, kappa_max
        a.tr_enabled, a.or_enabled = int(tr_enabled), int(or_enabled)
        a.rr_first, a.rr_prefix, a.rr_refresh = int(rr_first), int(rr_prefix), int(rr_refresh)
        return a

    def replan(self, cond_real, x_out, noise_remap, **kw):
        self._enter()
        a = self.replan_args(cond_real, x_out, noise_remap, **kw)
        info = abi.WamReplanInfo()
        self._check(self.lib.wam_replan(self.h, C.byref(a), C.byref(info)), "wam_replan")
        self._leave()
        return info

    def replan_begin(self, args):
        """Remap and enqueue the anticipatory prefix (args from replan_args)."""
        self._enter()
        self._check(self.lib.wam_replan_begin(self.h, C.byref(args)), "wam_replan_begin")

    def replan_end(self, args):
        self._enter()
        info = abi.WamReplanInfo()
        self._check(self.lib.wam_replan_end(self.h, C.byref(args), C.byref(info)), "wam_replan_end")
        self._leave()
        return info

    def set_option(self, option, value):
        self._check(self.lib.wam_set_option(self.h, option, int(value)), "wam_set_option")

    def sync(self):
        self._check(self.lib.wam_sync(self.h), "wam_sync")

    def profile_enable(self, kc, enable=True, max_launches=4096):
        self._check(self.lib.wam_profile_enable(self.h, kc, int(enable), max_launches), "wam_profile_enable")

    def profile_read(self, kc):
        t, n, w = C.c_double(), C.c_int64(), C.c_double()
        self._check(self.lib.wam_profile_read(self.h, kc, C.byref(t), C.byref(n), C.byref(w)), "wam_profile_read")
        return t.value, n.value, w.value


class IdmPair:
    """Independently executed video and action models (Sec. 3.3): per control
    step the video model's replan under the observation, then the action
    model's under the observation followed by the video model's new latent
    (packed on the device by wam_pack_condition).  Each model keeps its own
    replan state, schedule, RR decision and graphs."""

    def __init__(self, video: WamModel, action: WamModel, n_obs: int, c_obs: int):
        cv, ca = video.cfg, action.cfg
        if cv.Na != 0 or ca.Nv != 0 or ca.No != n_obs + cv.Nv or ca.Co < max(c_obs, cv.Cv):
            raise WamError("action condition must hold the observation and the video latent tokens")
        self.video, self.action = video, action
        self.n_obs, self.c_obs = n_obs, c_obs
        self.cond_action = torch.zeros((ca.B, ca.No, ca.Co), dtype=torch.float32, device=action.device)

    def replan(self, obs_real, x_video, x_action, noise_remap_video, noise_remap_action, video_kw=None,
               action_kw=None):
        """One control step; returns (video info, action info)."""
        iv = self.video.replan(obs_real, x_video, noise_remap_video, **(video_kw or {}))
        cv = self.video.cfg
        self.action.pack_condition(obs_real, self.n_obs, self.c_obs, x_video, cv.Nv, cv.Cv, self.video.traj,
                                   self.cond_action)
        ia = self.action.replan(self.cond_action, x_action, noise_remap_action, **(action_kw or {}))
        return iv, ia


def remap_noalloc(cfg: abi.WamConfig, x_bar, x_r, sigma_r, sigma_b0, shift_action, shift_video, noise, x_out,
                  stream: torch.cuda.Stream | None = None):
    """Trajectory Remapping without a handle or workspace (wam_remap_noalloc);
    enqueued on stream (default: torch's current stream on x_out's device)."""
    lib = abi.lib()
    s = stream if stream is not None else torch.cuda.current_stream(x_out.device)
    a = abi.WamRemapArgs(x_bar=_ptr(x_bar), x_r=_ptr(x_r), sigma_r=sigma_r, sigma_b0=sigma_b0,
                         shift_action=shift_action, shift_video=shift_video, noise=_ptr(noise), x_out=_ptr(x_out))
    rc = lib.wam_remap_noalloc(C.byref(cfg), C.byref(a), C.c_void_p(s.cuda_stream))
    if rc != abi.WAM_OK:
        raise WamError(f"wam_remap_noalloc: {lib.wam_status_string(rc).decode()}: "
                       f"{lib.wam_noalloc_last_error().decode()}")
    return x_out


# ---------------------------------------------------------------- layer operators
# stream: the call's stream (default: torch's current one), to which results that the
# call allocates belong, as under torch.cuda.stream(stream).
# There are no backward passes: a tensor that requires a gradient is refused, but under
# torch.no_grad.
FP8 = torch.float8_e4m3fn
_TYPES = {torch.float32: abi.WAM_FP32, torch.bfloat16: abi.WAM_BF16, FP8: abi.WAM_FP8}
_REAL = (torch.float32, torch.bfloat16)
_F32 = (torch.float32,)
_F8 = (FP8,)
_LAYOUTS = {"halves": abi.WAM_ROPE_HALVES, "pairs": abi.WAM_ROPE_PAIRS}
_NORMS = {"none": abi.WAM_NORM_NONE, "rms": abi.WAM_NORM_RMS, "layer": abi.WAM_NORM_LAYER}

# The argument structs as the C compiler lays them out (their ctypes twins in _lib):
# packing one takes a microsecond, filling its twin ten.
_ROPE_ARGS = struct.Struct("@10i4P12qPqP2Pf")
_NORM_ARGS = struct.Struct("@8i5P10q3P6q2P2f")
_QUANTIZE_ARGS = struct.Struct("@4iPqPqPq")
_MATMUL_ARGS = struct.Struct("@5iPqPqPqPqPPqPq")
_FP4_ARGS = struct.Struct("@3iPqPqPq")
_CACHE_ARGS = "4i4P12qPqi0P"  # the cache and its table, inside the calls' structs
_APPEND_ARGS = struct.Struct("@7i0P" + _CACHE_ARGS + "2P6q3PqPPd")
_ATTENTION_ARGS = struct.Struct("@5i0P" + _CACHE_ARGS + "P3qP3qP3q2PdPN")
_WORKSPACE = struct.Struct("@PN")  # at its end


def _operand(t, what, dtypes, index, shape=None):
    """Checks an operator's tensor: on GPU `index`, of one of dtypes, of the given
    shape, its last dimension contiguous."""
    if not isinstance(t, torch.Tensor) or t.get_device() != index:  # -1: not on a GPU
        raise WamError(f"{what}: needs a tensor on the GPU of the first operand")
    if t.dtype not in dtypes:
        raise WamError(f"{what}: dtype {t.dtype} is not supported")
    if shape is not None and t.shape != shape:
        raise WamError(f"{what}: shape {tuple(t.shape)} is not {tuple(shape)}")
    if not t.is_contiguous() and t.dim() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise WamError(f"{what}: the last dimension must be contiguous")
    if t.requires_grad and torch.is_grad_enabled():
        raise WamError(f"{what}: asks for a gradient, and the layer operators have none (detach it, or torch.no_grad)")
    return t


def _first(t, what, dtypes, dim):
    """Checks an operator's first tensor and returns the index of its GPU."""
    if not isinstance(t, torch.Tensor) or t.dim() != dim:
        raise WamError(f"{what}: needs a tensor of {dim} dimensions")
    if not t.is_cuda:
        raise WamError(f"{what}: libwam takes device tensors only")
    index = t.get_device()
    _operand(t, what, dtypes, index)
    return index


def _choice(table, key, what):
    try:
        return table[key]
    except (KeyError, TypeError):
        raise WamError(f"{what}: unknown value {key!r}") from None


def _new(stream, make, *args, **kw):
    """A new result of an operator on `stream`: memory of that stream's own, as another
    stream's may still be in use there."""
    if stream is None:
        return make(*args, **kw)
    with torch.cuda.stream(stream):
        return make(*args, **kw)


def _call(fn, args, index, stream, what):
    """Enqueues a handle-free operator on GPU `index` (stream: default torch's current one)."""
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(index)
    elif stream.device_index != index:
        raise WamError(f"{what}: stream of GPU {stream.device_index}, operands on GPU {index}")
    else:
        handle = stream.cuda_stream
    if index == torch._C._cuda_getDevice():
        rc = fn(args, handle)
    else:
        with torch.cuda.device(index):
            rc = fn(args, handle)
    if rc != abi.WAM_OK:
        raise WamError(f"{what}: {abi.lib().wam_status_string(rc).decode()}: "
                       f"{abi.lib().wam_noalloc_last_error().decode()}")


def _pack(form, what, *values):
    try:
        return form.pack(*values)
    except struct.error as e:
        raise WamError(f"{what}: {e}") from None


def _ptr_or_0(t):
    return 0 if t is None else t.data_ptr()


def rope_frequencies(sections, theta=10000.0, shared=False) -> np.ndarray:
    """Frequencies of the usual ladder for rope (wam_rope_frequencies): float64
    [sum(sections)], theta^(-j / n) along each axis of n pairs, or one ladder
    over all pairs."""
    if len(sections) != 3 or any(abs(n) > abi.WAM_MAX_HEAD for n in sections):  # ctypes cuts off what passes 32 bits
        raise WamError("rope_frequencies: needs three sections of at most WAM_MAX_HEAD pairs")
    sec = (C.c_int32 * 3)(*sections)
    freq = np.empty(min(max(sum(sec), 0), abi.WAM_MAX_HEAD // 2), np.float64)
    lib = abi.lib()
    rc = lib.wam_rope_frequencies(sec, theta, int(bool(shared)), freq.ctypes.data_as(C.POINTER(C.c_double)))
    if rc != abi.WAM_OK:
        raise WamError(f"wam_rope_frequencies: {lib.wam_noalloc_last_error().decode()}")
    return freq


_NO_HEADS = (0, 0, 0)


def rope(q, k, pos, sections, freq, *, layout="halves", q_gain=None, k_gain=None, eps=1e-6, q_out=None, k_out=None,
         stream: torch.cuda.Stream | None = None):
    """Rotary positions over up to three axes (wam_rope): q [B, T, Hq, dh] and k
    [B, T, Hk, dh] (or None), float32 or bfloat16, any strides with dh contiguous;
    pos float32 [T, 3] or [B, T, 3]; freq on the host, one value per pair.  With
    gains, float32 [dh], the per-head RMS norm comes first.  q_out / k_out: the
    results' buffers (q / k: in place; default: new ones).  Returns (q_out, k_out)."""
    index = _first(q, "rope: q", _REAL, 4)
    B, T, Hq, dh = q.shape
    own = (q.dtype,)
    Hk = 0
    if k is not None:
        _operand(k, "rope: k", own, index)
        if k.dim() != 4 or k.shape[0] != B or k.shape[1] != T or k.shape[3] != dh:
            raise WamError("rope: k must be [B, T, H, dh] as q")
        Hk = k.shape[2]
    each = isinstance(pos, torch.Tensor) and pos.dim() == 3  # sample has its own positions
    _operand(pos, "rope: pos", _F32, index, (B, T, 3) if each else (T, 3))
    if T > 1 and pos.stride(-2) != 3:
        raise WamError("rope: rows of pos must be contiguous")
    if len(sections) != 3 or len(freq) != sum(sections) or getattr(freq, "ndim", 1) != 1:
        raise WamError("rope: needs three sections and one frequency per pair")
    ladder = np.ascontiguousarray(freq, np.float64) if isinstance(freq, np.ndarray) else array("d", freq)
    at = ladder.ctypes.data if isinstance(ladder, np.ndarray) else ladder.buffer_info()[0]
    if q_gain is not None:
        _operand(q_gain, "rope: q_gain", _F32, index, (dh,))
    if k_gain is not None:
        _operand(k_gain, "rope: k_gain", _F32, index, (dh,))
    q_out = _new(stream, torch.empty_like, q) if q_out is None else _operand(q_out, "rope: q_out", own, index, q.shape)
    if k is not None:
        k_out = (_new(stream, torch.empty_like, k) if k_out is None else
                 _operand(k_out, "rope: k_out", own, index, k.shape))
    else:
        k_out = None
    ks, kos = (k.stride()[:3], k_out.stride()[:3]) if k is not None else (_NO_HEADS, _NO_HEADS)
    a = _pack(_ROPE_ARGS, "rope", B, T, Hq, Hk, dh, _TYPES[q.dtype], _choice(_LAYOUTS, layout, "rope: layout"),
              *sections, q.data_ptr(), _ptr_or_0(k), q_out.data_ptr(), _ptr_or_0(k_out), *q.stride()[:3], *ks,
              *q_out.stride()[:3], *kos, pos.data_ptr(), pos.stride(0) if each else 0, at,
              _ptr_or_0(q_gain), _ptr_or_0(k_gain), eps)
    _call(abi.lib().wam_rope, a, index, stream, "wam_rope")
    return q_out, k_out


def _row_vectors(v, what, index, B, T, D):
    """Pointer and strides (sample, row) of float32 vectors that broadcast to [B, T, D]."""
    if v is None:
        return 0, 0, 0
    _operand(v, what, _F32, index)
    own, n = v.shape, v.dim()
    b, t, d = own if n == 3 else (1, *own) if n == 2 else (1, 1, *own) if n == 1 else (0, 0, -1)
    if d != D or b not in (1, B) or t not in (1, T):
        raise WamError(f"{what}: shape {tuple(own)} does not broadcast to {(B, T, D)} with D values per row")
    s = v.stride()
    return v.data_ptr(), s[0] if b != 1 else 0, s[-2] if t != 1 else 0


_NO_ROWS = (0, 0)


def norm_residual(h, y=None, *, post="rms", post_gain=None, gate=None, res_scale=1.0, pre="layer", pre_gain=None,
                  scale=None, shift=None, eps=1e-6, h_out=None, u_dtype=None, u=None, u_scale=None,
                  stream: torch.cuda.Stream | None = None):
    """The norms around a block (wam_norm_residual), h and y [B, T, D] in float32 or
    bfloat16: h_out = res_scale h + gate post(y), u = pre(h_out) (1 + scale) + shift.
    post, pre: "none", "rms" or "layer"; pre None leaves u out.  gate, scale, shift:
    float32, anything that broadcasts to [B, T, D] with D contiguous; gains float32
    [D].  h_out: its buffer (h: in place; default: a new one).  u_dtype: float32,
    bfloat16 or float8_e4m3fn (default: that of u, else bfloat16).  Returns
    (h_out,), (h_out, u) or, for 8-bit blocks, (h_out, u, u_scale)."""
    index = _first(h, "norm_residual: h", _REAL, 3)
    shape = h.shape
    B, T, D = shape
    if y is not None:
        _operand(y, "norm_residual: y", _REAL, index, shape)
    if post_gain is not None:
        _operand(post_gain, "norm_residual: post_gain", _F32, index, (D,))
    if pre_gain is not None:
        _operand(pre_gain, "norm_residual: pre_gain", _F32, index, (D,))
    g, g0, g1 = _row_vectors(gate, "norm_residual: gate", index, B, T, D)
    c, c0, c1 = _row_vectors(scale, "norm_residual: scale", index, B, T, D)
    s, s0, s1 = _row_vectors(shift, "norm_residual: shift", index, B, T, D)
    h_out = (_new(stream, torch.empty_like, h) if h_out is None else
             _operand(h_out, "norm_residual: h_out", (h.dtype,), index, shape))
    post = _choice(_NORMS, post, "norm_residual: post")
    if pre is None:
        u = u_scale = None
        kind = u_type = 0
    else:
        kind = _choice(_NORMS, pre, "norm_residual: pre")
        if u is None:
            u = _new(stream, _new_rows, shape, torch.bfloat16 if u_dtype is None else u_dtype, h.device,
                     "norm_residual: u_dtype", h)
        else:
            _operand(u, "norm_residual: u", tuple(_TYPES) if u_dtype is None else (u_dtype,), index, shape)
        u_type = _TYPES[u.dtype]
        if u_type == abi.WAM_FP8:
            blocks = (B, T, -(-D // 128))
            u_scale = (_new(stream, torch.empty, blocks, dtype=torch.float32, device=h.device) if u_scale is None else
                       _operand(u_scale, "norm_residual: u_scale", _F32, index, blocks))
        else:
            u_scale = None
    rows = lambda t: _NO_ROWS if t is None else t.stride()[:2]  # noqa: E731
    a = _pack(_NORM_ARGS, "norm_residual", B, T, D, _TYPES[h.dtype], 0 if y is None else _TYPES[y.dtype], u_type, post,
              kind, h.data_ptr(), _ptr_or_0(y), h_out.data_ptr(), _ptr_or_0(u), _ptr_or_0(u_scale), *rows(h), *rows(y),
              *rows(h_out), *rows(u), *rows(u_scale), g, c, s, g0, g1, c0, c1, s0, s1, _ptr_or_0(post_gain),
              _ptr_or_0(pre_gain), res_scale, eps)
    _call(abi.lib().wam_norm_residual, a, index, stream, "wam_norm_residual")
    return (h_out,) if u is None else (h_out, u) if u_scale is None else (h_out, u, u_scale)


def _new_rows(shape, dtype, dev, what, like=None):
    """A new tensor; e4m3 rows start a multiple of 16 bytes apart, as matmul_fp8
    takes them.  like: a tensor of that shape (empty_like is the faster call)."""
    if dtype not in _TYPES:
        raise WamError(f"{what}: dtype {dtype} is not supported")
    if dtype != FP8 or shape[-1] % 16 == 0:
        if like is not None and like.is_contiguous():
            return torch.empty_like(like, dtype=dtype)
        return torch.empty(shape, dtype=dtype, device=dev)
    padded = (*shape[:-1], -(-shape[-1] // 16) * 16)
    return torch.empty(padded, dtype=dtype, device=dev)[..., :shape[-1]]


def quantize_fp8(x, *, block_rows=1, q=None, scale=None, stream: torch.cuda.Stream | None = None):
    """8-bit blocks (wam_quantize_fp8) of x [M, K], float32 or bfloat16: block_rows 1
    for activations (1 x 128), 128 for weights (128 x 128).  Returns (q, scale):
    float8_e4m3fn [M, K] with rows a multiple of 16 bytes apart and float32
    [ceil(M / block_rows), ceil(K / 128)]; x stands for q * scale."""
    index = _first(x, "quantize_fp8: x", _REAL, 2)
    if block_rows not in (1, 128):
        raise WamError("quantize_fp8: block_rows must be 1 or 128")
    M, K = x.shape
    if q is None:
        q = _new(stream, _new_rows, (M, K), FP8, x.device, "quantize_fp8: q")
    else:
        _operand(q, "quantize_fp8: q", _F8, index, x.shape)
    shape = (-(-M // block_rows), -(-K // 128))
    scale = (_new(stream, torch.empty, shape, dtype=torch.float32, device=x.device) if scale is None else
             _operand(scale, "quantize_fp8: scale", _F32, index, shape))
    a = _pack(_QUANTIZE_ARGS, "quantize_fp8", M, K, _TYPES[x.dtype], block_rows, x.data_ptr(), x.stride(0), q.data_ptr(),
              q.stride(0), scale.data_ptr(), scale.stride(0))
    _call(abi.lib().wam_quantize_fp8, a, index, stream, "wam_quantize_fp8")
    return q, scale


def matmul_fp8(a, a_scale, w, w_scale, *, bias=None, gelu=False, out=None, out_dtype=None, out_scale=None,
               stream: torch.cuda.Stream | None = None):
    """out [M, N] = act((a * a_scale) (w * w_scale)^T + bias) of 8-bit blocks
    (wam_matmul_fp8): a [M, K] with scales per row and 128 columns, w [N, K] with
    scales per 128 x 128, both as quantize_fp8 gives them (a block's two scales are
    multiplied first, in float32); rows are read up to the next multiple of 16 bytes,
    what lies there does not enter.  bias float32 [N]; gelu: the tanh form.
    out float32, bfloat16 (default: a new bfloat16 one) or
    float8_e4m3fn: then returns (out, out_scale), blocks for the next product."""
    index = _first(a, "matmul_fp8: a", _F8, 2)
    _operand(w, "matmul_fp8: w", _F8, index)
    M, K = a.shape
    if w.dim() != 2 or w.shape[1] != K:
        raise WamError("matmul_fp8: needs a [M, K] and w [N, K]")
    N, kb = w.shape[0], -(-K // 128)
    _operand(a_scale, "matmul_fp8: a_scale", _F32, index, (M, kb))
    _operand(w_scale, "matmul_fp8: w_scale", _F32, index, (-(-N // 128), kb))
    if bias is not None:
        _operand(bias, "matmul_fp8: bias", _F32, index, (N,))
    if out is None:
        out = _new(stream, _new_rows, (M, N), torch.bfloat16 if out_dtype is None else out_dtype, a.device,
                   "matmul_fp8: out_dtype")
    else:
        _operand(out, "matmul_fp8: out", tuple(_TYPES) if out_dtype is None else (out_dtype,), index, (M, N))
    kind = _TYPES[out.dtype]
    scale_at = scale_stride = 0
    if kind == abi.WAM_FP8:
        shape = (M, -(-N // 128))
        out_scale = (_new(stream, torch.empty, shape, dtype=torch.float32, device=a.device) if out_scale is None else
                     _operand(out_scale, "matmul_fp8: out_scale", _F32, index, shape))
        scale_at, scale_stride = out_scale.data_ptr(), out_scale.stride(0)
    args = _pack(_MATMUL_ARGS, "matmul_fp8", M, N, K, kind, abi.WAM_ACT_GELU if gelu else abi.WAM_ACT_NONE,
                 a.data_ptr(), a.stride(0), a_scale.data_ptr(), a_scale.stride(0), w.data_ptr(), w.stride(0),
                 w_scale.data_ptr(), w_scale.stride(0), _ptr_or_0(bias), out.data_ptr(), out.stride(0), scale_at,
                 scale_stride)
    _call(abi.lib().wam_matmul_fp8, args, index, stream, "wam_matmul_fp8")
    return (out, out_scale) if kind == abi.WAM_FP8 else out


_U8 = (torch.uint8,)
_I32 = (torch.int32,)


def _matrix(M, n, dtype, dev):
    """A new matrix (the fastest call for one)."""
    return torch.empty_strided((M, n), (n, 1), dtype=dtype, device=dev)


def _byte_rows(M, n, dev, unit):
    """A new matrix of bytes whose rows start a multiple of `unit` bytes apart."""
    wide = -(-n // unit) * unit
    x = _matrix(M, wide, torch.uint8, dev)
    return x if wide == n else x.as_strided((M, n), (wide, 1))


def quantize_fp4(x, *, q=None, scale=None, stream: torch.cuda.Stream | None = None):
    """4-bit blocks of 32 columns (wam_quantize_fp4) of x [M, K], float32 or bfloat16.
    Returns (q, scale): uint8 [M, ceil(K / 2)], two codes a byte, and uint8
    [M, ceil(K / 32)], a power of two each, with rows as matmul_fp4 takes them (a
    multiple of 16 and 4 bytes apart)."""
    index = _first(x, "quantize_fp4: x", _REAL, 2)
    M, K = x.shape
    codes, blocks = (M, -(-K // 2)), (M, -(-K // 32))
    q = (_new(stream, _byte_rows, *codes, x.device, 16) if q is None else
         _operand(q, "quantize_fp4: q", _U8, index, codes))
    scale = (_new(stream, _byte_rows, *blocks, x.device, 4) if scale is None else
             _operand(scale, "quantize_fp4: scale", _U8, index, blocks))
    a = _pack(_FP4_ARGS, "quantize_fp4", M, K, _TYPES[x.dtype], x.data_ptr(), x.stride(0), q.data_ptr(), q.stride(0),
              scale.data_ptr(), scale.stride(0))
    _call(abi.lib().wam_quantize_fp4, a, index, stream, "wam_quantize_fp4")
    return q, scale


def dequantize_fp4(q, scale, *, columns=None, dtype=None, out=None, stream: torch.cuda.Stream | None = None):
    """The values that 4-bit blocks stand for (wam_dequantize_fp4): q [M, n] and scale
    [M, ceil(columns / 32)] as quantize_fp4 gives them; columns: 2 n (the default), or
    2 n - 1 where the last code is none.  dtype: bfloat16 (the default) or float32 of
    a new result, [M, columns]."""
    index = _first(q, "dequantize_fp4: q", _U8, 2)
    M, n = q.shape
    K = 2 * n if columns is None else columns
    if K not in (2 * n, 2 * n - 1) or K < 0:
        raise WamError("dequantize_fp4: columns must be twice those of q, or one less")
    _operand(scale, "dequantize_fp4: scale", _U8, index, (M, -(-K // 32)))
    if out is None:
        dtype = torch.bfloat16 if dtype is None else dtype
        if dtype not in _REAL:
            raise WamError(f"dequantize_fp4: dtype {dtype} is not supported")
        out = _new(stream, _matrix, M, K, dtype, q.device)
    else:
        _operand(out, "dequantize_fp4: out", _REAL if dtype is None else (dtype,), index, (M, K))
    a = _pack(_FP4_ARGS, "dequantize_fp4", M, K, _choice(_TYPES, out.dtype, "dequantize_fp4: dtype"), q.data_ptr(),
              q.stride(0), scale.data_ptr(), scale.stride(0), out.data_ptr(), out.stride(0))
    _call(abi.lib().wam_dequantize_fp4, a, index, stream, "wam_dequantize_fp4")
    return out


def matmul_fp4(a, a_scale, w, w_scale, *, bias=None, gelu=False, out=None, out_dtype=None, out_scale=None,
               stream: torch.cuda.Stream | None = None):
    """out [M, N] = act(a w^T + bias) of matrices in 4-bit blocks (wam_matmul_fp4): codes a
    [M, n] and w [N, n] with their scales [M or N, ceil(n / 16)], as quantize_fp4 gives
    them (each byte of a row is two values: an odd last one has a zero beside it); rows
    are read up to the next multiple of 16 bytes (scales: of 4), what lies there does not
    enter.  bias float32 [N]; gelu: the tanh form.  out: float32, bfloat16 (default: a
    new bfloat16 one); uint8 asks for 4-bit blocks of the result: then returns
    (out [M, ceil(N / 2)], out_scale [M, ceil(N / 32)]) for the next product."""
    index = _first(a, "matmul_fp4: a", _U8, 2)
    _operand(w, "matmul_fp4: w", _U8, index)
    M, n = a.shape
    if w.dim() != 2 or w.shape[1] != n:
        raise WamError("matmul_fp4: needs a and w with the same number of columns")
    N, kb = w.shape[0], -(-n // 16)
    _operand(a_scale, "matmul_fp4: a_scale", _U8, index, (M, kb))
    _operand(w_scale, "matmul_fp4: w_scale", _U8, index, (N, kb))
    if bias is not None:
        _operand(bias, "matmul_fp4: bias", _F32, index, (N,))
    kind = torch.bfloat16 if out is None and out_dtype is None else out_dtype if out is None else out.dtype
    blocks = kind == torch.uint8
    if not blocks and kind not in _REAL:
        raise WamError(f"matmul_fp4: out_dtype {kind} is not supported")
    shape = (M, -(-N // 2)) if blocks else (M, N)
    if out is None:
        out = (_new(stream, _byte_rows, *shape, a.device, 16) if blocks else
               _new(stream, _matrix, *shape, kind, a.device))
    else:
        _operand(out, "matmul_fp4: out", (kind,) if out_dtype is None else (out_dtype,), index, shape)
    scale_at = scale_stride = 0
    if blocks:
        shape = (M, -(-N // 32))
        out_scale = (_new(stream, _byte_rows, *shape, a.device, 4) if out_scale is None else
                     _operand(out_scale, "matmul_fp4: out_scale", _U8, index, shape))
        scale_at, scale_stride = out_scale.data_ptr(), out_scale.stride(0)
    args = _pack(_MATMUL_ARGS, "matmul_fp4", M, N, 2 * n, abi.WAM_FP4 if blocks else _TYPES[kind],
                 abi.WAM_ACT_GELU if gelu else abi.WAM_ACT_NONE, a.data_ptr(), a.stride(0), a_scale.data_ptr(),
                 a_scale.stride(0), w.data_ptr(), w.stride(0), w_scale.data_ptr(), w_scale.stride(0), _ptr_or_0(bias),
                 out.data_ptr(), out.stride(0), scale_at, scale_stride)
    _call(abi.lib().wam_matmul_fp4, args, index, stream, "wam_matmul_fp4")
    return (out, out_scale) if blocks else out


class KvCache(NamedTuple):
    """Keys and values of a layer in 4-bit blocks, in pages of tokens: codes uint8
    [pages, page, H, dh / 2] and scales uint8 [pages, page, H, dh / 32], any strides
    with a head contiguous (a plain tuple of the four does too)."""
    k: torch.Tensor
    k_scale: torch.Tensor
    v: torch.Tensor
    v_scale: torch.Tensor


def new_kv_cache(pages, page, heads, dh, device="cuda:0") -> KvCache:
    """A KvCache of zeros whose pages hold a head's tokens side by side, as
    cache_attention reads them fastest."""
    if dh % 32 or min(pages, page, heads, dh) < 0:
        raise WamError("new_kv_cache: sizes must be >= 0, heads whole blocks of 32")
    make = lambda n: torch.zeros((pages, heads, page, n), dtype=torch.uint8, device=device).transpose(1, 2)  # noqa: E731
    return KvCache(make(dh // 2), make(dh // 32), make(dh // 2), make(dh // 32))


def _cache_part(t, what, index, shape):
    """Strides of page, token and head of one of a cache's tensors."""
    if not isinstance(t, torch.Tensor) or t.get_device() != index or t.dtype is not torch.uint8 or t.shape != shape:
        raise WamError(f"{what}: the cache needs uint8 tensors on the GPU of the first operand, codes [pages, page, H, "
                       "dh / 2] and scales [pages, page, H, dh / 32]")
    page, token, head, step = t.stride()
    if step != 1 and shape[3] > 1 and t.numel() > 0:
        raise WamError(f"{what}: a head of the cache must be contiguous")
    return page, token, head


def _cache_values(cache, table, index, B, H, dh, what):
    """A cache and its page table as the calls' structs hold them."""
    if not isinstance(cache, tuple) or len(cache) != 4:
        raise WamError(f"{what}: cache must be a KvCache")
    k, k_scale, v, v_scale = cache
    shape = k.shape if isinstance(k, torch.Tensor) else ()
    if len(shape) != 4 or (H is not None and shape[2] != H) or 2 * shape[3] != dh:
        raise WamError(f"{what}: the cache's codes must be [pages, page, H, dh / 2]")
    pages, page, H, half = shape
    scales = (pages, page, H, half // 16)
    _operand(table, f"{what}: table", _I32, index)
    if table.dim() != 2 or table.shape[0] != B:
        raise WamError(f"{what}: table must be [B, pages of a sequence]")
    ks, kss = _cache_part(k, what, index, shape), _cache_part(k_scale, what, index, scales)
    vs, vss = _cache_part(v, what, index, shape), _cache_part(v_scale, what, index, scales)
    return (pages, page, H, dh, k.data_ptr(), k_scale.data_ptr(), v.data_ptr(), v_scale.data_ptr(), *ks, *kss, *vs, *vss,
            table.data_ptr(), table.stride(0), table.shape[1])


def _per_sequence(t, what, index, B):
    """Pointer of int32 [B] or None."""
    if t is None:
        return 0
    _operand(t, what, _I32, index, (B,))
    return t.data_ptr()


def cache_append(cache, k, v, table, start, *, rows=None, pos=None, sections=(0, 0, 0), freq=(), layout="halves",
                 k_gain=None, eps=1e-6, stream: torch.cuda.Stream | None = None):
    """Appends new rows' keys and values to a paged cache in 4-bit blocks
    (wam_cache_append), in place: k, v [B, T, H, dh], float32 or bfloat16, any strides
    with dh contiguous; row t of sequence b becomes token start[b] + t, which lies in
    page table[b, token // page] (table int32 [B, n], start int32 [B]; an entry that is no
    page drops its tokens).  rows int32 [B]: only the first rows[b] of a sequence count.
    Keys first get the RMS norm with k_gain, float32 [dh], and the rotary positions pos
    float32 [T, 3] or [B, T, 3], sections, freq and layout of rope.  Returns cache."""
    index = _first(k, "cache_append: k", _REAL, 4)
    B, T, H, dh = k.shape
    _operand(v, "cache_append: v", (k.dtype,), index, k.shape)
    held = _cache_values(cache, table, index, B, H, dh, "cache_append")
    _operand(start, "cache_append: start", _I32, index, (B,))
    count = _per_sequence(rows, "cache_append: rows", index, B)
    if len(sections) != 3 or len(freq) != sum(sections) or getattr(freq, "ndim", 1) != 1:
        raise WamError("cache_append: needs three sections and one frequency per pair")
    ladder = np.ascontiguousarray(freq, np.float64) if isinstance(freq, np.ndarray) else array("d", freq)
    at = ladder.ctypes.data if isinstance(ladder, np.ndarray) else ladder.buffer_info()[0]
    pos_at = pos_stride = 0
    if pos is not None:
        each = isinstance(pos, torch.Tensor) and pos.dim() == 3  # sample has its own positions
        _operand(pos, "cache_append: pos", _F32, index, (B, T, 3) if each else (T, 3))
        if T > 1 and pos.stride(-2) != 3:
            raise WamError("cache_append: rows of pos must be contiguous")
        pos_at, pos_stride = pos.data_ptr(), pos.stride(0) if each else 0
    if k_gain is not None:
        _operand(k_gain, "cache_append: k_gain", _F32, index, (dh,))
    a = _pack(_APPEND_ARGS, "cache_append", B, T, _TYPES[k.dtype], _choice(_LAYOUTS, layout, "cache_append: layout"),
              *sections, *held, k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3], start.data_ptr(), count,
              pos_at, pos_stride, at, _ptr_or_0(k_gain), eps)
    _call(abi.lib().wam_cache_append, a, index, stream, "wam_cache_append")
    return cache


def cache_attention(q, cache, table, lengths, *, rows=None, causal=False, scale=None, out=None, lse=None,
                    stream: torch.cuda.Stream | None = None):
    """Attention of new rows over a paged cache in 4-bit blocks (wam_cache_attention): q
    [B, T, Hq, dh], float32 or bfloat16, any strides with dh contiguous, Hq a multiple of
    the cache's heads; sequence b has lengths[b] tokens (int32 [B]) in the pages of
    table[b] (int32 [B, n]; an entry that is no page leaves its tokens out).  causal: the
    last tokens are the rows' own, and row t sees those up to its own.  rows int32 [B]:
    only the first rows[b] of a sequence count, the others' results are 0, as are those
    of rows that see no token.  scale: default 1 / sqrt(dh).  Returns out, of q's shape
    and type; lse: a float32 [B, T, Hq] buffer for the logarithm of each row's sum.  The
    call is planned by the table's width: table[:, :n] with the pages that the longest
    sequence needs is faster than one of a whole context."""
    index = _first(q, "cache_attention: q", _REAL, 4)
    B, T, Hq, dh = q.shape
    held = _cache_values(cache, table, index, B, None, dh, "cache_attention")
    _operand(lengths, "cache_attention: lengths", _I32, index, (B,))
    count = _per_sequence(rows, "cache_attention: rows", index, B)
    out = (_new(stream, torch.empty_strided, q.shape, (T * Hq * dh, Hq * dh, dh, 1), dtype=q.dtype, device=q.device)
           if out is None else
           _operand(out, "cache_attention: out", (q.dtype,), index, q.shape))
    lse_stride = _NO_HEADS
    if lse is not None:
        _operand(lse, "cache_attention: lse", _F32, index, (B, T, Hq))
        lse_stride = lse.stride()
    head = (B, T, Hq, _TYPES[q.dtype], int(bool(causal)), *held, q.data_ptr(), *q.stride()[:3], out.data_ptr(),
            *out.stride()[:3], _ptr_or_0(lse), *lse_stride, lengths.data_ptr(), count,
            1.0 / math.sqrt(dh) if scale is None and dh else scale)
    lib = abi.lib()
    a = _pack(_ATTENTION_ARGS, "cache_attention", *head, 0, 0)
    need = lib.wam_cache_attention_workspace(a)
    if need:
        # freed to the call's own stream when this returns: later work there may take it
        work = _new(stream, _matrix, 1, need, torch.uint8, q.device)
        a = a[:-_WORKSPACE.size] + _WORKSPACE.pack(work.data_ptr(), need)
    _call(lib.wam_cache_attention, a, index, stream, "wam_cache_attention")
    return out


def probe_mfma_bf16(shape: int = 0, n_blocks: int = 1024, iters: int = 20000, device="cuda:0"):
    """Achievable bf16 MFMA rate (wam_probe_mfma_bf16): returns (TFLOP/s, ms)."""
    lib = abi.lib()
    sink = torch.empty(n_blocks * 256, dtype=torch.float32, device=device)
    stream = C.c_void_p(torch.cuda.current_stream(sink.device).cuda_stream)
    tf, ms = C.c_double(), C.c_double()
    rc = lib.wam_probe_mfma_bf16(stream, shape, n_blocks, iters, _ptr(sink), C.byref(tf), C.byref(ms))
    if rc != abi.WAM_OK:
        raise WamError(f"wam_probe_mfma_bf16: {lib.wam_status_string(rc).decode()}")
    return tf.value, ms.value


def probe_copy(nbytes: int = 1 << 30, reps: int = 5, device="cuda:0"):
    """Achievable streaming copy rate (wam_probe_copy): returns (GB/s counting
    read + write bytes, ms per copy)."""
    lib = abi.lib()
    n = nbytes // 4
    src = torch.ones(n, dtype=torch.float32, device=device)
    dst = torch.empty_like(src)
    stream = C.c_void_p(torch.cuda.current_stream(src.device).cuda_stream)
    gbs, ms = C.c_double(), C.c_double()
    rc = lib.wam_probe_copy(stream, _ptr(src), _ptr(dst), n * 4, reps, C.byref(gbs), C.byref(ms))
    if rc != abi.WAM_OK:
        raise WamError(f"wam_probe_copy: {lib.wam_status_string(rc).decode()}")
    return gbs.value, ms.value
