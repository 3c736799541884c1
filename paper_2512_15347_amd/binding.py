"""ctypes binding of libprogrpo.so: same names as the C ABI, argument marshalling only.

PyTorch appears here for device memory and streams; every step of the sampling path runs inside
the HIP library.  There is no CPU fallback: importing this module without the built library
raises.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("PROGRPO_LIB", os.path.join(_HERE, "libprogrpo.so"))

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
        "(there is no fallback path)")

_lib = C.CDLL(LIB_PATH)

PG_OK, PG_EINVAL, PG_ESHAPE, PG_ENAN, PG_ESCHED, PG_EWORKSPACE, PG_EHIP = range(7)
STATUS_NAMES = ["PG_OK", "PG_EINVAL", "PG_ESHAPE", "PG_ENAN", "PG_ESCHED", "PG_EWORKSPACE", "PG_EHIP"]
PG_SAMPLER_FLOW, PG_SAMPLER_DDIM, PG_SAMPLER_TABLE = 0, 1, 2
PG_NET_NONE, PG_NET_ADALN, PG_NET_CROSS, PG_NET_JOINT, PG_NET_MMDIT = 0, 1, 2, 3, 4

WEIGHT_IDS = ["pe_w", "pe_b", "pos", "t_w1", "t_b1", "t_w2", "t_b2", "ctx_w", "ctx_b", "fmod_w", "fmod_b",
              "f_w", "f_b", "mod_w", "mod_b", "qkv_w", "qkv_b", "o_w", "o_b", "fc1_w", "fc1_b", "fc2_w",
              "fc2_b", "cq_w", "cq_b", "ckv_w", "ckv_b", "co_w", "co_b",
              "c_mod_w", "c_mod_b", "c_qkv_w", "c_qkv_b", "c_o_w", "c_o_b", "c_fc1_w", "c_fc1_b", "c_fc2_w", "c_fc2_b",
              "qn_g", "kn_g", "c_qn_g", "c_kn_g"]
FIRST_BLOCK_ID = WEIGHT_IDS.index("mod_w")

_dp = C.POINTER(C.c_double)
_ip = C.POINTER(C.c_int32)


class pg_config(C.Structure):
    _fields_ = [("P", C.c_int32), ("N", C.c_int32), ("C", C.c_int32), ("H", C.c_int32), ("W", C.c_int32),
                ("T", C.c_int32), ("sampler_kind", C.c_int32), ("noise_level", C.c_double),
                ("eta", C.c_double), ("beta0", C.c_double), ("beta1", C.c_double), ("T_train", C.c_int32),
                ("tab_A", _dp), ("tab_B", _dp), ("tab_C", _dp), ("tab_P", _dp), ("tab_Q", _dp), ("tab_tin", _dp),
                ("net_kind", C.c_int32), ("D", C.c_int32), ("blocks", C.c_int32), ("heads", C.c_int32),
                ("Lc", C.c_int32), ("Dc", C.c_int32), ("n_sched", C.c_int32),
                ("sched_group", _ip), ("sched_step", _ip), ("sched_k", _ip),
                ("probe_bias", C.c_double), ("adv_eps", C.c_double)]


class pg_buffers(C.Structure):
    _fields_ = [("x", C.c_void_p * 2), ("u", C.c_void_p), ("orig_id", C.c_void_p * 2),
                ("group_offsets", C.c_void_p), ("group_of", C.c_void_p), ("rewards", C.c_void_p),
                ("masks", C.c_void_p), ("sel_idx", C.c_void_p), ("logp_hist", C.c_void_p),
                ("logp_sum", C.c_void_p), ("adv", C.c_void_p), ("probe_w", C.c_void_p),
                ("weights", C.c_void_p), ("ctx", C.c_void_p), ("y", C.c_void_p), ("status", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("x_hist", C.c_void_p)]


class pg_cache(C.Structure):
    _fields_ = [("layers", C.c_int32), ("n_pages", C.c_int32), ("heads", C.c_int32), ("page", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("width", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("refs", C.c_void_p), ("status", C.c_void_p)]


class pg_logits(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("stride", C.c_int64), ("dtype", C.c_int32), ("rows", C.c_int32),
                ("vocab", C.c_int32), ("tokens_stride", C.c_int32), ("tokens", C.c_void_p), ("n_prompt", C.c_void_p),
                ("n_tokens", C.c_void_p), ("repetition", C.c_void_p), ("frequency", C.c_void_p), ("presence", C.c_void_p),
                ("bias_offsets", C.c_void_p), ("bias_ids", C.c_void_p), ("bias_values", C.c_void_p),
                ("n_bias", C.c_int32), ("n_masks", C.c_int32), ("allow", C.c_void_p), ("allow_row", C.c_void_p)]


class PgError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < 7 else status}: {message}")
        self.status = status


_vp, _i32, _i64, _u64, _u32, _f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_uint32, C.c_double
_cp, _lp = C.POINTER(pg_cache), C.POINTER(pg_logits)
_SIGNATURES = {
    "pg_last_error": (C.c_char_p, []),
    "pg_create": (_i32, [C.POINTER(pg_config), C.POINTER(_vp)]),
    "pg_destroy": (None, [_vp]),
    "pg_workspace_bytes": (C.c_size_t, [_vp]),
    "pg_weights_numel": (_i64, [_vp]),
    "pg_weight_slot": (_i32, [_vp, _i32, _i32, C.POINTER(_i64), _ip, _ip, _ip]),
    "pg_get_tables": (_i32, [_vp, _dp, _dp, _dp, _dp, _dp, _dp]),
    "pg_get_schedule": (_i32, [_vp, _i32, _ip, _ip]),
    "pg_bind": (_i32, [_vp, C.POINTER(pg_buffers)]),
    "pg_state": (_i32, [_vp, _ip, _ip, _ip, _ip, C.POINTER(_i64), C.POINTER(_i64)]),
    "pg_init_group": (_i32, [_vp, _u64, _vp]),
    "pg_net_forward": (_i32, [_vp, _i32, _vp]),
    "pg_prune": (_i32, [_vp, _i32, _vp]),
    "pg_prune_forced": (_i32, [_vp, _i32, C.POINTER(_u64), _vp, _vp]),
    "pg_step": (_i32, [_vp, _i32, _vp]),
    "pg_advantages": (_i32, [_vp, _vp]),
    "pg_sample_group": (_i32, [_vp, _u64, _vp]),
    "pg_check": (_i32, [_vp, _vp]),
    "pg_policy_ratio": (_i32, [_vp, _vp, _f64, _vp, _vp, _vp, _vp]),
    "pg_select_final": (_i32, [_vp, _i32, _ip, _u32, _vp]),
    "pg_init_latents": (_i32, [_vp, _vp, _i64, _i64, _u64, _vp]),
    "pg_step_scratch_floats": (_i64, [_i64, _i64]),
    "pg_sde_step_logprob": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _f64, _f64, _f64, _u64,
                                    _u32, _vp, _vp]),
    "pg_sde_step_logprob_bf16": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _f64, _f64, _f64, _u64,
                                         _u32, _vp, _vp]),
    "pg_preview_reward": (_i32, [_vp, _vp, _vp, _vp, _i64, _i64, _f64, _f64, _f64, _vp, _vp]),
    "pg_ovf_scratch_ints": (_i64, [_i64]),
    "pg_ovf_select": (_i32, [_vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "pg_ovf_select_noalloc": (_i32, [_vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp]),
    "pg_ovf_select_large": (_i32, [_vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "pg_uniform_select": (_i32, [_vp, _vp, _i32, _u64, _u32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "pg_group_stats": (_i32, [_vp, _vp, _i32, _f64, _vp, _vp, _vp]),
    "pg_compact_gather": (_i32, [_vp, _vp, _vp, _i64, _i64, _vp]),
    "pg_group_advantages": (_i32, [_vp, _vp, _i32, _f64, _vp, _vp]),
    "pg_gemm_bf16": (_i32, [_vp, _i64, _vp, _i64, _vp, _vp, _i64, _i64, _i64, _i64, _vp]),
    "pg_gemm_tile": (_i32, [_i64, _i64, _i64, _i32]),
    "pg_gemm_bf16_tile": (_i32, [_vp, _i64, _vp, _i64, _vp, _vp, _i64, _i64, _i64, _i64, _i32, _i32, _vp]),
    "pg_attention_bf16": (_i32, [_vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _vp]),
    "pg_attention_kernel": (_i32, [_i32] * 5),
    "pg_attention_network": (_i32, [_vp, _vp, _vp, _vp] + [_i32] * 7 + [_vp]),
    "pg_mfma_probe": (_i32, [_i32, _i32, C.c_float, _vp, _dp, _vp]),
    "pg_cache_clear": (_i32, [_cp, _vp]),
    "pg_cache_reserve": (_i32, [_cp, _vp, _vp, _vp, _vp, _i32, _vp]),
    "pg_cache_append": (_i32, [_cp, _i32, _vp, _vp, _i64, _vp, _vp, _vp, _i32, _i32, _vp]),
    "pg_cache_scratch_ints": (_i64, [_cp, _i32]),
    "pg_cache_select": (_i32, [_cp, _vp, _vp, _i32, _vp, _vp, _vp, _i32, _vp, _vp]),
    "pg_cache_compact": (_i32, [_cp, _vp, _vp, _i32, _vp, _vp]),
    "pg_cache_check": (_i32, [_cp, _vp]),
    "pg_paged_attention_workspace": (C.c_size_t, [_cp, _i32, _i32, _i32]),
    "pg_paged_attention": (_i32, [_cp, _i32, _vp, _i64, _vp, _i32, _vp, _vp, _i32, _i32, _f64, _i32, _vp, _i64, _vp, _vp,
                                  C.c_size_t, _vp]),
    "pg_logits_adjust": (_i32, [_lp, _vp, _i64, _vp]),
    "pg_sample_scratch_floats": (_i64, [_i32, _i32]),
    "pg_sample_tokens": (_i32, [_lp, _vp, _u64, _u32, _vp, _vp, _vp, _vp, _vp]),
    "pg_logprob_scratch_floats": (_i64, [_i32, _i32, _i32]),
    "pg_token_logprobs": (_i32, [_lp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp]),
    "pg_token_logprobs_backward": (_i32, [_lp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp]),
    "pg_distill_scratch_floats": (_i64, [_i32, _i32]),
    "pg_distill_loss": (_i32, [_lp, _vp, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp]),
    "pg_distill_backward": (_i32, [_lp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _i64, _vp]),
    "pg_surrogate_scratch_floats": (_i64, [_i32, _i32]),
    "pg_token_surrogate": (_i32, [_vp] * 6 + [_i32] * 3 + [_f64] * 3 + [_vp] * 6),
    "pg_profile_begin": (_i32, [_i32]),
    "pg_profile_read": (_i32, [_i32, _dp, _dp, C.POINTER(_i64)]),
    "pg_profile_end": (_i32, []),
}
EXPORTS = sorted(_SIGNATURES)
for _name, (_res, _args) in _SIGNATURES.items():
    _fn = getattr(_lib, _name)          # AttributeError here = symbol missing from the library
    _fn.restype = _res
    _fn.argtypes = _args


def pg_last_error():
    return _lib.pg_last_error().decode()


def _check(status):
    if status != PG_OK:
        raise PgError(status, pg_last_error())


def _ptr(t):
    """Device (or host) address of a torch tensor / None."""
    if t is None or isinstance(t, int):
        return t
    assert t.is_contiguous(), "the C ABI takes contiguous buffers"
    return t.data_ptr()


_current_stream = None


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    global _current_stream
    if _current_stream is None:
        import torch
        # the handle alone, without the stream object around it, which costs more than the launch of a small kernel; torch keeps this
        # function to itself
        device, raw = torch.cuda.current_device, getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _current_stream = (lambda: raw(device())) if raw else (lambda: torch.cuda.current_stream().cuda_stream)
    return _current_stream()


# ---------------------------------------------------------------- context-level calls

def make_config(cfg, probe_bias=0.0, adv_eps=1e-6, net=True, tables=None):
    """workloads-style dict -> (pg_config, keep-alive list)."""
    keep = []
    c = pg_config()
    for f in ("P", "N", "C", "H", "W", "T"):
        setattr(c, f, int(cfg[f]))
    s = cfg["sampler"]
    if tables is not None:
        c.sampler_kind = PG_SAMPLER_TABLE
        for name, key in (("tab_A", "A"), ("tab_B", "B"), ("tab_C", "C"), ("tab_P", "P"), ("tab_Q", "Q"),
                          ("tab_tin", "t_in")):
            arr = (C.c_double * cfg["T"])(*[float(v) for v in tables[key]])
            keep.append(arr)
            setattr(c, name, C.cast(arr, _dp))
    elif s["kind"] == "flow":
        c.sampler_kind = PG_SAMPLER_FLOW
        c.noise_level = float(s["a"])
    else:
        c.sampler_kind = PG_SAMPLER_DDIM
        c.eta, c.beta0, c.beta1, c.T_train = float(s["eta"]), float(s["beta0"]), float(s["beta1"]), int(s["T_train"])
    if net:
        c.net_kind = {"adaln": PG_NET_ADALN, "cross": PG_NET_CROSS, "joint": PG_NET_JOINT,
                      "mmdit": PG_NET_MMDIT}[cfg["kind"]]
        c.D, c.blocks, c.heads, c.Lc, c.Dc = (int(cfg[k]) for k in ("D", "blocks", "heads", "Lc", "Dc"))
    else:
        c.net_kind = PG_NET_NONE
    entries = [(g, st, k) for g, lst in enumerate(cfg["schedule"]) for (st, k) in lst]
    c.n_sched = len(entries)
    if entries:
        for name, col in (("sched_group", 0), ("sched_step", 1), ("sched_k", 2)):
            arr = (C.c_int32 * len(entries))(*[int(e[col]) for e in entries])
            keep.append(arr)
            setattr(c, name, C.cast(arr, _ip))
    c.probe_bias = float(probe_bias)
    c.adv_eps = float(adv_eps)
    return c, keep


def pg_create(config):
    out = _vp()
    _check(_lib.pg_create(C.byref(config), C.byref(out)))
    return out


def pg_destroy(ctx):
    _lib.pg_destroy(ctx)


def pg_workspace_bytes(ctx):
    return int(_lib.pg_workspace_bytes(ctx))


def pg_weights_numel(ctx):
    return int(_lib.pg_weights_numel(ctx))


def pg_weight_slot(ctx, wid, block=0):
    off, rows, cols, ld = _i64(), _i32(), _i32(), _i32()
    _check(_lib.pg_weight_slot(ctx, wid, block, C.byref(off), C.byref(rows), C.byref(cols), C.byref(ld)))
    return off.value, rows.value, cols.value, ld.value


def pg_get_tables(ctx, T):
    arrs = [(C.c_double * T)() for _ in range(6)]
    _check(_lib.pg_get_tables(ctx, *arrs))
    return {k: np.array(a[:]) for k, a in zip(("A", "B", "C", "P", "Q", "t_in"), arrs)}


def pg_get_schedule(ctx, step, P):
    k, off = (C.c_int32 * P)(), (C.c_int32 * (P + 1))()
    _check(_lib.pg_get_schedule(ctx, step, k, off))
    return list(k), list(off)


def pack_weights(ctx, cfg, weights):
    """Lay the network tensors out as the library asks (uint16 bf16 bit patterns, host array)."""
    from .workloads import bf16_bits
    flat = np.zeros(pg_weights_numel(ctx), dtype=np.uint16)

    def put(wid, block, arr):
        off, rows, cols, ld = pg_weight_slot(ctx, wid, block)
        a = np.asarray(arr, dtype=np.float32).reshape(rows, cols)
        view = flat[off:off + rows * ld].reshape(rows, ld)
        view[:, :cols] = bf16_bits(a)

    for wid, name in enumerate(WEIGHT_IDS):
        if wid < FIRST_BLOCK_ID:
            if name in weights:
                put(wid, 0, weights[name])
        else:
            for b, blk in enumerate(weights["blocks"]):
                if name in blk:
                    put(wid, b, blk[name])
    return flat


class Buffers:
    """Device tensors for one context (torch owns the memory) + the filled pg_buffers."""

    def __init__(self, ctx, cfg, inputs=None, weights_flat=None, device="cuda:0", keep_history=False):
        import torch
        P, N, T, d = cfg["P"], cfg["N"], cfg["T"], cfg["d"]
        M0 = P * N
        dev = torch.device(device)
        z = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device=dev)
        self.x = [z(M0, d), z(M0, d)]
        self.u = z(M0, d)
        self.orig_id = [z(M0, dtype=torch.int32), z(M0, dtype=torch.int32)]
        self.group_offsets = z(P + 1, dtype=torch.int32)
        self.group_of = z(M0, dtype=torch.int32)
        self.rewards = z(M0)
        self.masks = z(P, dtype=torch.int64)
        self.sel_idx = z(M0, dtype=torch.int32)
        self.logp_hist = z(T, M0)
        self.logp_sum = z(M0)
        self.adv = z(M0)
        self.status = z(4, dtype=torch.int32)
        self.probe_w = (torch.from_numpy(np.ascontiguousarray(inputs["probe_w"], dtype=np.float32)).to(dev)
                        if inputs is not None else z(d))
        self.weights = self.ctx_tok = self.y = None
        if weights_flat is not None:
            self.weights = torch.from_numpy(weights_flat.view(np.int16)).to(dev)
            self.y = torch.from_numpy(np.ascontiguousarray(inputs["y"], dtype=np.float32)).to(dev)
            if inputs.get("ctx") is not None:
                from .workloads import bf16_bits
                self.ctx_tok = torch.from_numpy(bf16_bits(inputs["ctx"]).view(np.int16)).to(dev)
        nbytes = pg_workspace_bytes(ctx)
        self.workspace = torch.empty(max(nbytes, 256) + 256, dtype=torch.uint8, device=dev)
        ws_ptr = (self.workspace.data_ptr() + 255) & ~255
        b = pg_buffers()
        b.x[0], b.x[1] = self.x[0].data_ptr(), self.x[1].data_ptr()
        b.u = self.u.data_ptr()
        b.orig_id[0], b.orig_id[1] = self.orig_id[0].data_ptr(), self.orig_id[1].data_ptr()
        for name in ("group_offsets", "group_of", "rewards", "masks", "sel_idx", "logp_hist", "logp_sum", "adv",
                     "probe_w", "status"):
            setattr(b, name, getattr(self, name).data_ptr())
        b.weights = _ptr(self.weights)
        b.ctx = _ptr(self.ctx_tok)
        b.y = _ptr(self.y)
        b.workspace = ws_ptr
        b.workspace_bytes = nbytes
        self.x_hist = z(T + 1, M0, d) if keep_history else None
        b.x_hist = _ptr(self.x_hist)
        self.c = b


def pg_bind(ctx, buffers):
    _check(_lib.pg_bind(ctx, C.byref(buffers.c if isinstance(buffers, Buffers) else buffers)))


def pg_state(ctx, P):
    M, cx, ci, ev, up = _i32(), _i32(), _i32(), _i64(), _i64()
    off = (C.c_int32 * (P + 1))()
    _check(_lib.pg_state(ctx, C.byref(M), C.byref(cx), C.byref(ci), off, C.byref(ev), C.byref(up)))
    return dict(M=M.value, cur_x=cx.value, cur_id=ci.value, offsets=list(off), evals=ev.value, updates=up.value)


def pg_init_group(ctx, seed, stream=None):
    _check(_lib.pg_init_group(ctx, seed, _stream(stream)))


def pg_net_forward(ctx, step, stream=None):
    _check(_lib.pg_net_forward(ctx, step, _stream(stream)))


def pg_prune(ctx, step, stream=None):
    _check(_lib.pg_prune(ctx, step, _stream(stream)))


def pg_prune_forced(ctx, step, masks, ovf_masks_out=None, stream=None):
    arr = (C.c_uint64 * len(masks))(*[int(m) for m in masks])
    _check(_lib.pg_prune_forced(ctx, step, arr, _ptr(ovf_masks_out), _stream(stream)))


def pg_step(ctx, step, stream=None):
    _check(_lib.pg_step(ctx, step, _stream(stream)))


def pg_advantages(ctx, stream=None):
    _check(_lib.pg_advantages(ctx, _stream(stream)))


def pg_sample_group(ctx, seed, stream=None):
    _check(_lib.pg_sample_group(ctx, seed, _stream(stream)))


SELECT_OVF, SELECT_UNIFORM = 0, 1


def pg_select_final(ctx, mode, k_per_group, draw=0, stream=None):
    k = (C.c_int32 * len(k_per_group))(*[int(v) for v in k_per_group])
    _check(_lib.pg_select_final(ctx, mode, k, draw, _stream(stream)))


def pg_policy_ratio(ctx, weights_new, clip_eps, logp_new, ratio, J, stream=None):
    _check(_lib.pg_policy_ratio(ctx, _ptr(weights_new), clip_eps, _ptr(logp_new), _ptr(ratio), _ptr(J), _stream(stream)))


def pg_check(ctx, stream=None):
    _check(_lib.pg_check(ctx, _stream(stream)))


# ---------------------------------------------------------------- kernel-level calls

def pg_init_latents(x, orig_id, seed, stream=None):
    n, d = x.shape
    _check(_lib.pg_init_latents(_ptr(x), _ptr(orig_id), n, d, seed, _stream(stream)))


def pg_step_scratch_floats(n_traj, d):
    return int(_lib.pg_step_scratch_floats(n_traj, d))


def pg_sde_step_logprob(x, u, x_out, logp, logp_hist, logp_sum, src, orig_id, n_traj, d, A, B, Cc, seed, step,
                        partials, stream=None):
    _check(_lib.pg_sde_step_logprob(_ptr(x), _ptr(u), _ptr(x_out), _ptr(logp), _ptr(logp_hist), _ptr(logp_sum),
                                    _ptr(src), _ptr(orig_id), n_traj, d, A, B, Cc, seed, step, _ptr(partials),
                                    _stream(stream)))


def pg_sde_step_logprob_bf16(x, u, x_out, logp, logp_hist, logp_sum, src, orig_id, n_traj, d, A, B, Cc, seed, step,
                             partials, stream=None):
    _check(_lib.pg_sde_step_logprob_bf16(_ptr(x), _ptr(u), _ptr(x_out), _ptr(logp), _ptr(logp_hist), _ptr(logp_sum),
                                         _ptr(src), _ptr(orig_id), n_traj, d, A, B, Cc, seed, step, _ptr(partials),
                                         _stream(stream)))


def pg_preview_reward(x, u, w, rewards, n_traj, d, Pc, Qc, bias, partials, stream=None):
    _check(_lib.pg_preview_reward(_ptr(x), _ptr(u), _ptr(w), _ptr(rewards), n_traj, d, Pc, Qc, bias,
                                  _ptr(partials), _stream(stream)))


def pg_ovf_scratch_ints(n_groups):
    return int(_lib.pg_ovf_scratch_ints(n_groups))


def pg_ovf_select(rewards, group_offsets, k, n_groups, masks, sel_idx, new_offsets, status, scratch, stream=None):
    _check(_lib.pg_ovf_select(_ptr(rewards), _ptr(group_offsets), _ptr(k), n_groups, _ptr(masks), _ptr(sel_idx),
                              _ptr(new_offsets), _ptr(status), _ptr(scratch), _stream(stream)))


PG_OVF_NOALLOC_MAX_GROUPS = 4194304


def pg_ovf_select_noalloc(rewards, group_offsets, k, n_groups, masks, sel_idx, new_offsets, status, stream=None):
    _check(_lib.pg_ovf_select_noalloc(_ptr(rewards), _ptr(group_offsets), _ptr(k), n_groups, _ptr(masks), _ptr(sel_idx),
                                      _ptr(new_offsets), _ptr(status), _stream(stream)))


def pg_ovf_select_large(rewards, group_offsets, k, n_groups, mask_words, masks, sel_idx, new_offsets, status, scratch,
                        stream=None):
    _check(_lib.pg_ovf_select_large(_ptr(rewards), _ptr(group_offsets), _ptr(k), n_groups, mask_words, _ptr(masks),
                                    _ptr(sel_idx), _ptr(new_offsets), _ptr(status), _ptr(scratch), _stream(stream)))


def pg_uniform_select(group_offsets, k, n_groups, seed, draw, masks, sel_idx, new_offsets, status, scratch, stream=None):
    _check(_lib.pg_uniform_select(_ptr(group_offsets), _ptr(k), n_groups, seed, draw, _ptr(masks), _ptr(sel_idx),
                                  _ptr(new_offsets), _ptr(status), _ptr(scratch), _stream(stream)))


def pg_group_stats(rewards, group_offsets, n_groups, delta, sigma, clustered_share, stream=None):
    _check(_lib.pg_group_stats(_ptr(rewards), _ptr(group_offsets), n_groups, delta, _ptr(sigma), _ptr(clustered_share),
                               _stream(stream)))


def pg_compact_gather(x, out, src, n_out, d, stream=None):
    _check(_lib.pg_compact_gather(_ptr(x), _ptr(out), _ptr(src), n_out, d, _stream(stream)))


def pg_group_advantages(rewards, group_offsets, n_groups, eps, adv, stream=None):
    _check(_lib.pg_group_advantages(_ptr(rewards), _ptr(group_offsets), n_groups, eps, _ptr(adv), _stream(stream)))


def pg_gemm_bf16(A, lda, W, ldw, bias, Cout, ldc, M, N, K, stream=None):
    _check(_lib.pg_gemm_bf16(_ptr(A), lda, _ptr(W), ldw, _ptr(bias), _ptr(Cout), ldc, M, N, K, _stream(stream)))


def pg_gemm_tile(M, N, K, accumulate=False):
    return int(_lib.pg_gemm_tile(M, N, K, int(accumulate)))


def pg_gemm_bf16_tile(A, lda, W, ldw, bias, Cout, ldc, M, N, K, accumulate=False, tile=0, stream=None):
    _check(_lib.pg_gemm_bf16_tile(_ptr(A), lda, _ptr(W), ldw, _ptr(bias), _ptr(Cout), ldc, M, N, K, int(accumulate), tile, _stream(stream)))


def pg_attention_bf16(q, k, vt, out, B, Lq, Lk, heads, hd, stream=None):
    _check(_lib.pg_attention_bf16(_ptr(q), _ptr(k), _ptr(vt), _ptr(out), B, Lq, Lk, heads, hd, _stream(stream)))


def pg_attention_kernel(B, Lq, Lk, heads, hd):
    return int(_lib.pg_attention_kernel(B, Lq, Lk, heads, hd))


def pg_attention_network(q, k, vt, out, B, Lq, Lk, Lk_pad, heads, hd, kernel=0, stream=None):
    _check(_lib.pg_attention_network(_ptr(q), _ptr(k), _ptr(vt), _ptr(out), B, Lq, Lk, Lk_pad, heads, hd, kernel, _stream(stream)))


# ---------------------------------------------------------------- rollouts of a token policy

PG_CACHE_BF16, PG_CACHE_E4M3 = 0, 1
PG_CACHE_MAX_ROWS = 16384
PG_LOGITS_F32, PG_LOGITS_BF16 = 0, 1


class _Types:
    """torch's type objects, looked up once: comparing them costs a tenth of comparing their names."""

    def __getattr__(self, name):
        import torch
        self.int32, self.float32, self.bfloat16 = torch.int32, torch.float32, torch.bfloat16
        # what is read as bf16 and as codes, the bits alone among them
        self.pairs = frozenset((torch.bfloat16, torch.int16, torch.uint16))
        self.codes = frozenset((torch.float8_e4m3fn, torch.int8, torch.uint8))
        return self.__dict__[name]


_types = _Types()


def _wanted(t, kind, shape):
    raise AssertionError(f"a contiguous {kind} tensor of shape {shape} is wanted: {t.dtype} {tuple(t.shape)}, strides {t.stride()}")


def _i32s(t, *shape):
    """Address of a contiguous int32 tensor of this shape, or None."""
    if t is None:
        return None
    if t.dtype is not _types.int32 or t.shape != shape or not t.is_contiguous():
        _wanted(t, "int32", shape)
    return t.data_ptr()


def _f32s(t, *shape):
    if t is None:
        return None
    if t.dtype is not _types.float32 or t.shape != shape or not t.is_contiguous():
        _wanted(t, "float32", shape)
    return t.data_ptr()


def _rows(t, heads, head_dim):
    """Address and row stride (in elements) of [rows, heads, head_dim] in bf16 whose rows may be slices of longer ones."""
    rows, n, d = t.shape
    s0, s1, s2 = t.stride()
    assert n == heads and d == head_dim and (t.dtype is _types.bfloat16 or t.dtype in _types.pairs) and s2 == 1 and (s1 == d or n == 1), \
        f"[rows, {heads}, {head_dim}] in bf16 with contiguous heads wanted: {t.dtype} {tuple(t.shape)}, strides {t.stride()}"
    return t.data_ptr(), s0 if rows > 1 else max(s0, n * d)


class Cache:
    """Device tensors of a paged cache (the caller's) + the filled pg_cache.

    k: [layers, pages, heads, page, head_dim], v: [layers, pages, heads, head_dim, page], both bf16 (or 16-bit integers: its bits) or
    e4m3 codes (or 8-bit integers); refs: int32 [pages]; width: entries of a table's row."""

    def __init__(self, k, v, refs, width, k_scale=None, v_scale=None, status=None):
        import torch
        layers, n_pages, heads, page, head_dim = k.shape
        assert tuple(v.shape) == (layers, n_pages, heads, head_dim, page)
        assert any(k.dtype in kind and v.dtype in kind for kind in (_types.pairs, _types.codes)), f"pools of {k.dtype} and {v.dtype}"
        self.k, self.v, self.refs, self.k_scale, self.v_scale = k, v, refs, k_scale, v_scale
        self.status = torch.zeros(4, dtype=torch.int32, device=k.device) if status is None else status
        c = pg_cache()
        c.layers, c.n_pages, c.heads, c.page, c.head_dim, c.width = layers, n_pages, heads, page, head_dim, width
        c.dtype = PG_CACHE_BF16 if k.element_size() == 2 else PG_CACHE_E4M3
        c.k, c.v = _ptr(k), _ptr(v)
        c.k_scale, c.v_scale = _f32s(k_scale, layers, heads), _f32s(v_scale, layers, heads)
        c.refs, c.status = _i32s(refs, n_pages), _i32s(self.status, 4)
        self.c, self.ref = c, C.byref(c)
        self.heads, self.head_dim, self.width = heads, head_dim, width

    @classmethod
    def create(cls, layers, n_pages, heads, page, head_dim, width, dtype=PG_CACHE_BF16, device="cuda:0"):
        """A cache with all pages free; e4m3 codes with scales of 1 to be overwritten."""
        import torch
        kind = torch.bfloat16 if dtype == PG_CACHE_BF16 else torch.uint8
        z = lambda *shape, dtype=kind: torch.zeros(*shape, dtype=dtype, device=device)
        scales = (None, None) if dtype == PG_CACHE_BF16 else (z(layers, heads, dtype=torch.float32) + 1, z(layers, heads, dtype=torch.float32) + 1)
        return cls(z(layers, n_pages, heads, page, head_dim), z(layers, n_pages, heads, head_dim, page), z(n_pages, dtype=torch.int32), width, *scales)


def pg_cache_clear(cache, stream=None):
    _check(_lib.pg_cache_clear(cache.ref, _stream(stream)))


def pg_cache_reserve(cache, table, lens, add, lens_out, stream=None):
    n = lens.shape[0]
    _check(_lib.pg_cache_reserve(cache.ref, _i32s(table, n, cache.width), _i32s(lens, n), _i32s(add, n), _i32s(lens_out, n), n, _stream(stream)))


def pg_cache_append(cache, layer, k_new, v_new, table, lens, cu=None, stream=None):
    n, tokens = lens.shape[0], k_new.shape[0]
    k, ks = _rows(k_new, cache.heads, cache.head_dim)
    v, vs = _rows(v_new, cache.heads, cache.head_dim)
    assert v_new.shape[0] == tokens and (ks == vs or tokens < 2), "keys and values of the same number and stride"
    _check(_lib.pg_cache_append(cache.ref, layer, k, v, ks, _i32s(table, n, cache.width), _i32s(lens, n), _i32s(cu, n + 1), n, tokens,
                                _stream(stream)))


def pg_cache_scratch_ints(cache, n_rows):
    return int(_lib.pg_cache_scratch_ints(cache.ref, n_rows))


def pg_cache_select(cache, table_in, lens_in, src, table_out, lens_out, scratch, stream=None):
    n, m, w = lens_in.shape[0], src.shape[0], cache.width
    assert scratch.numel() >= pg_cache_scratch_ints(cache, max(n, m))
    _check(_lib.pg_cache_select(cache.ref, _i32s(table_in, n, w), _i32s(lens_in, n), n, _i32s(src, m), _i32s(table_out, m, w),
                                _i32s(lens_out, m), m, _i32s(scratch, scratch.shape[0]), _stream(stream)))


def pg_cache_compact(cache, table, lens, scratch, stream=None):
    n = lens.shape[0]
    assert scratch.numel() >= pg_cache_scratch_ints(cache, 0)
    _check(_lib.pg_cache_compact(cache.ref, _i32s(table, n, cache.width), _i32s(lens, n), n, _i32s(scratch, scratch.shape[0]), _stream(stream)))


def pg_cache_check(cache, stream=None):
    _check(_lib.pg_cache_check(cache.ref, _stream(stream)))


def pg_paged_attention_workspace(cache, n_q, heads_q, max_len):
    return int(_lib.pg_paged_attention_workspace(cache.ref, n_q, heads_q, max_len))


def pg_paged_attention(cache, layer, q, table, lens, out, max_len, workspace=None, lse=None, row_of=None, scale=0.0, stream=None):
    n, heads, hd = q.shape
    rows = table.shape[0]
    qp, qs = _rows(q, heads, cache.head_dim)
    op, os_ = _rows(out, heads, cache.head_dim)
    assert out.shape[0] == n
    wp, size = (None, 0) if workspace is None else (_ptr(workspace), workspace.numel() * workspace.element_size())
    _check(_lib.pg_paged_attention(cache.ref, layer, qp, qs, _i32s(table, rows, cache.width), rows, _i32s(row_of, n), _i32s(lens, n), n,
                                   heads, scale, max_len, op, os_, _f32s(lse, n, heads), wp, size, _stream(stream)))


class Logits:
    """Logits [rows, vocab] (fp32 or bf16; rows may be slices of longer ones), what is to be done to them, and the filled pg_logits.
    It is a handle: the tensors' contents may change between calls."""

    def __init__(self, logits, tokens=None, n_prompt=None, n_tokens=None, repetition=None, frequency=None, presence=None,
                 bias_offsets=None, bias_ids=None, bias_values=None, allow=None, allow_row=None):
        rows, vocab = logits.shape
        assert str(logits.dtype) in ("torch.float32", "torch.bfloat16") and (vocab == 1 or logits.stride(1) == 1)
        self.keep = (logits, tokens, n_prompt, n_tokens, repetition, frequency, presence, bias_offsets, bias_ids, bias_values, allow, allow_row)
        d = pg_logits()
        d.logits, d.stride = logits.data_ptr(), logits.stride(0) if rows > 1 else max(logits.stride(0), vocab)
        d.dtype = PG_LOGITS_F32 if logits.element_size() == 4 else PG_LOGITS_BF16
        d.rows, d.vocab = rows, vocab
        d.tokens_stride = 0 if tokens is None else tokens.shape[1]
        d.tokens = _i32s(tokens, rows, d.tokens_stride)
        d.n_prompt, d.n_tokens = _i32s(n_prompt, rows), _i32s(n_tokens, rows)
        d.repetition, d.frequency, d.presence = (_f32s(t, rows) for t in (repetition, frequency, presence))
        d.bias_offsets = _i32s(bias_offsets, rows + 1)
        d.n_bias = 0 if bias_ids is None else bias_ids.shape[0]
        d.bias_ids, d.bias_values = _i32s(bias_ids, d.n_bias), _f32s(bias_values, d.n_bias)
        d.n_masks = 0 if allow is None else allow.shape[0]
        d.allow = _i32s(allow, d.n_masks, (vocab + 31) // 32)
        d.allow_row = _i32s(allow_row, rows)
        self.c, self.ref, self.rows, self.vocab = d, C.byref(d), rows, vocab
        self.scratch = pg_sample_scratch_floats(rows, vocab)
        self.loss_scratch = {}                               # floats, by what they are for


def pg_logits_adjust(desc, out, stream=None):
    rows, vocab = desc.rows, desc.vocab
    s0, s1 = out.stride()
    if out.shape != (rows, vocab) or out.dtype is not _types.float32 or (vocab > 1 and s1 != 1):
        _wanted(out, "float32", (rows, vocab))
    _check(_lib.pg_logits_adjust(desc.ref, out.data_ptr(), s0 if rows > 1 else max(s0, vocab), _stream(stream)))


def pg_sample_scratch_floats(rows, vocab):
    return int(_lib.pg_sample_scratch_floats(rows, vocab))


def pg_sample_tokens(desc, temperature, seed, step, ids, token, logp, scratch, stream=None):
    n = desc.rows
    assert scratch.numel() * scratch.element_size() >= 4 * desc.scratch
    _check(_lib.pg_sample_tokens(desc.ref, _f32s(temperature, n), seed, step, _i32s(ids, n), _i32s(token, n), _f32s(logp, n), _ptr(scratch),
                                 _stream(stream)))


# ---------------------------------------------------------------- what a token policy learns from

PG_TOP_MAX, PG_DISTILL_MAX = 64, 256
PG_LOGPROB_STATS, PG_DISTILL_STATS = 4, 8
PG_DISTILL_TOP, PG_DISTILL_TAIL = 0, 1


def _gradient(desc, d_logits):
    """Address and row stride of the gradient of desc's logits, which has their type."""
    rows, vocab = desc.rows, desc.vocab
    s0, s1 = d_logits.stride()
    if d_logits.shape != (rows, vocab) or d_logits.dtype is not desc.keep[0].dtype or (vocab > 1 and s1 != 1):
        _wanted(d_logits, str(desc.keep[0].dtype), (rows, vocab))
    return d_logits.data_ptr(), s0 if rows > 1 else max(s0, vocab)


def _scratch(scratch, floats):
    """Address of a scratch tensor of at least so many floats (may be None for 0)."""
    if floats and (scratch is None or not scratch.is_contiguous() or scratch.numel() * scratch.element_size() < 4 * floats):
        raise AssertionError(f"scratch of {floats} floats wanted")
    return None if scratch is None else scratch.data_ptr()


def _loss_scratch(desc, scratch, top=None):
    """The same for a call on these logits, of `top` alternatives (None: of a distillation)."""
    floats = desc.loss_scratch.get(top)
    if floats is None:
        floats = pg_distill_scratch_floats(desc.rows, desc.vocab) if top is None else pg_logprob_scratch_floats(desc.rows, desc.vocab, top)
        desc.loss_scratch[top] = floats
    return _scratch(scratch, floats)


def pg_logprob_scratch_floats(rows, vocab, n_top=0):
    return int(_lib.pg_logprob_scratch_floats(rows, vocab, n_top))


def pg_token_logprobs(desc, target, logp, scratch, temperature=None, entropy=None, stats=None, top_ids=None, top_logp=None, stream=None):
    n = desc.rows
    top = 0 if top_ids is None and top_logp is None else (top_logp if top_ids is None else top_ids).shape[1]
    _check(_lib.pg_token_logprobs(desc.ref, _f32s(temperature, n), _i32s(target, n), _f32s(logp, n), _f32s(entropy, n),
                                  _f32s(stats, n, PG_LOGPROB_STATS), top, _i32s(top_ids, n, top), _f32s(top_logp, n, top),
                                  _loss_scratch(desc, scratch, top), _stream(stream)))


def pg_token_logprobs_backward(desc, target, stats, d_logits, g_logp=None, g_entropy=None, temperature=None, stream=None):
    n = desc.rows
    to, stride = _gradient(desc, d_logits)
    _check(_lib.pg_token_logprobs_backward(desc.ref, _f32s(temperature, n), _i32s(target, n), _f32s(stats, n, PG_LOGPROB_STATS), _f32s(g_logp, n),
                                           _f32s(g_entropy, n), to, stride, _stream(stream)))


def pg_distill_scratch_floats(rows, vocab):
    return int(_lib.pg_distill_scratch_floats(rows, vocab))


def pg_distill_loss(desc, teacher_ids, teacher_logp, loss, scratch, tail=False, temperature=None, stats=None, stream=None):
    n, k = desc.rows, teacher_ids.shape[1]
    _check(_lib.pg_distill_loss(desc.ref, _f32s(temperature, n), PG_DISTILL_TAIL if tail else PG_DISTILL_TOP, _i32s(teacher_ids, n, k),
                                _f32s(teacher_logp, n, k), k, _f32s(loss, n), _f32s(stats, n, PG_DISTILL_STATS),
                                _loss_scratch(desc, scratch), _stream(stream)))


def pg_distill_backward(desc, teacher_ids, teacher_logp, stats, g_loss, d_logits, temperature=None, stream=None):
    n, k = desc.rows, teacher_ids.shape[1]
    to, stride = _gradient(desc, d_logits)
    _check(_lib.pg_distill_backward(desc.ref, _f32s(temperature, n), _i32s(teacher_ids, n, k), _f32s(teacher_logp, n, k), k,
                                    _f32s(stats, n, PG_DISTILL_STATS), _f32s(g_loss, n), to, stride, _stream(stream)))


def pg_surrogate_scratch_floats(n_seq, max_len):
    return int(_lib.pg_surrogate_scratch_floats(n_seq, max_len))


def pg_token_surrogate(logp, logp_old, adv, cu, objective, g_logp, clip_low, clip_high, max_len, scratch=None, logp_ref=None, kl_coef=0.0,
                       weight=None, kl=None, clipped=None, stream=None):
    n, tokens = adv.shape[0], logp.shape[0]
    _check(_lib.pg_token_surrogate(_f32s(logp, tokens), _f32s(logp_old, tokens), _f32s(logp_ref, tokens), _f32s(adv, n), _f32s(weight, n),
                                   _i32s(cu, n + 1), n, tokens, max_len, clip_low, clip_high, kl_coef, _f32s(objective, n), _f32s(kl, n),
                                   _i32s(clipped, n), _f32s(g_logp, tokens), _scratch(scratch, pg_surrogate_scratch_floats(n, max_len)),
                                   _stream(stream)))


def pg_mfma_probe(blocks, iters, operand_scale, out, stream=None):
    flops = C.c_double()
    _check(_lib.pg_mfma_probe(blocks, iters, operand_scale, _ptr(out), C.byref(flops), _stream(stream)))
    return flops.value


def pg_profile_begin(max_records=1 << 16):
    _check(_lib.pg_profile_begin(max_records))


def pg_profile_read(kind):
    ms, work, n = C.c_double(), C.c_double(), _i64()
    _check(_lib.pg_profile_read(kind, C.byref(ms), C.byref(work), C.byref(n)))
    return dict(ms=ms.value, work=work.value, launches=n.value)


def pg_profile_end():
    _check(_lib.pg_profile_end())
