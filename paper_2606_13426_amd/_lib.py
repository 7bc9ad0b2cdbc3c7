"""ctypes binding of libspecdiff.so (include/specdiff.h), same names as the C ABI.

Argument marshalling only: torch tensors are passed as device pointers with
their element strides, the stream is torch's current stream, and every status
other than SD_OK raises SpecDiffError with sd_last_error().  There is no
fallback: if the library has not been built, loading raises.
"""
import ctypes
import os
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspecdiff.so")

SD_OK, SD_EINVAL, SD_EHIP, SD_EUNSUPPORTED, SD_ENOMEM, SD_ENUMERIC = 0, -1, -2, -3, -4, -5
SD_BLOCK, SD_TOKEN = 0, 1
SD_FP32, SD_BF16 = 0, 1
SD_USAMPLE_EXACT, SD_USAMPLE_PAPER = 0, 1
SD_RESIDUAL_DECOMPOSITION, SD_RESIDUAL_REFLECTION = 0, 1
SD_DRAFTER_FREE, SD_DRAFTER_FROZEN = 0, 1
SD_TYPE_F32, SD_TYPE_BF16, SD_TYPE_F16 = 0, 1, 2
SD_ROPE_PAIRS, SD_ROPE_HALVES = 0, 1
SD_TREE_IID, SD_TREE_DISTINCT, SD_TREE_GIVEN = 0, 1, 2
SD_MAX_BLOCK = 64
SD_MAX_TREE = 64
SD_MAX_TOP, SD_MAX_VOCAB = 32, 1 << 24
TAG_INIT, TAG_DRAFT, TAG_COIN, TAG_USAMPLE, TAG_RESID, TAG_TARGET = 1, 2, 3, 4, 5, 6

c_int32, c_int64, c_uint32, c_uint64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64
c_double, c_size_t, c_void_p, c_char_p = ctypes.c_double, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_char_p


class sd_schedule(ctypes.Structure):
    _fields_ = [("n_steps", c_int32), ("beta_min", c_double), ("beta_max", c_double),
                ("churn", c_double)]


class sd_stride(ctypes.Structure):
    _fields_ = [("chain", c_int64), ("row", c_int64)]


class sd_stride_h(ctypes.Structure):
    _fields_ = [("seq", c_int64), ("row", c_int64), ("head", c_int64)]


class sd_stats(ctypes.Structure):
    _fields_ = [("rounds", c_int64), ("chain_rounds", c_int64), ("steps", c_int64),
                ("ties", c_int64), ("mean_tau", c_double), ("finished", c_int32),
                ("groups", c_int32), ("tau_hist", c_int64 * (SD_MAX_BLOCK + 2))]


class sd_sampler_options(ctypes.Structure):
    _fields_ = [("mode", c_int32), ("usample_mode", c_int32), ("residual", c_int32),
                ("drafter", c_int32), ("omega", c_double), ("start_round", c_int32),
                ("max_rounds", c_int32), ("groups", c_int32)]


class sd_sampler_view(ctypes.Structure):
    _fields_ = [("x", c_void_p), ("y", c_void_p), ("cache", c_void_p), ("cache_step", c_void_p),
                ("k", c_void_p), ("round", c_void_p), ("mq", c_void_p), ("lrp", c_void_p),
                ("n_tiles", c_int32), ("tau", c_void_p), ("coins", c_void_p),
                ("log_alpha_res", c_void_p), ("u", c_void_p), ("ties", c_void_p)]


class sd_kernel_stat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("launches", c_int64), ("total_ms", c_double)]


class SpecDiffError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"status {status}: {msg}")
        self.status = status


P = c_void_p
S = sd_stride
SH = sd_stride_h
# (name, restype, argtypes) of every exported function, in header order
SIGNATURES = [
    ("sd_abi_version", c_int32, []),
    ("sd_last_error", c_char_p, []),
    ("sd_schedule_table", c_int32, [ctypes.POINTER(sd_schedule), P]),
    ("sd_target_create", c_int32, [ctypes.POINTER(sd_schedule), c_int32, c_int32, P, P, P, c_int32,
                                   ctypes.POINTER(c_void_p)]),
    ("sd_target_destroy", c_int32, [P]),
    ("sd_target_mean_workspace", c_size_t, [P, c_int32]),
    ("sd_target_mean", c_int32, [P, c_int32, P, c_int64, P, P, c_int64, P, c_int64, P, c_size_t, P]),
    ("sd_target_mean_noalloc", c_int32, [P, c_int32, P, c_int64, P, P, c_int64, P, c_int64, P]),
    ("sd_target_mean_noalloc_max_bytes", c_size_t, []),
    ("sd_init_chains", c_int32, [c_int32, c_int32, c_uint64, P, P]),
    ("sd_draft_block", c_int32, [ctypes.POINTER(sd_schedule), c_int32, c_int32, c_int32, P, P, P, P,
                                 c_uint64, P, S, P, S, P]),
    ("sd_verify_block", c_int32, [c_int32, c_int32, c_int32, c_int32, P, S, P, S, P, S, P, P, P,
                                  c_uint64, c_int32, P, P, P, P, P, P, P]),
    ("sd_verify_block_tempered", c_int32, [c_int32, c_int32, c_int32, c_int32, c_double, P, S, P, S, P,
                                           S, P, P, P, c_uint64, c_int32, P, P, P, P, P, P, P]),
    ("sd_sample_residual", c_int32, [c_int32, c_int32, c_int32, P, S, P, S, P, S, P, P, P, P, P, P, P,
                                     c_uint64, P, P]),
    ("sd_sample_residual_reflection", c_int32, [c_int32, c_int32, c_int32, P, S, P, S, P, S, P, P, P, P,
                                                P, c_uint64, P, P]),
    ("sd_sampler_workspace", c_size_t, [P, c_int32, c_int32]),
    ("sd_run_sampler", c_int32, [P, c_int32, c_int32, c_int32, c_int32, c_uint64, P, P, c_int32,
                                 ctypes.POINTER(sd_stats), P, c_size_t, P]),
    ("sd_run_sampler_ex", c_int32, [P, c_int32, c_int32, ctypes.POINTER(sd_sampler_options), c_uint64, P,
                                    P, c_int32, ctypes.POINTER(sd_stats), P, c_size_t, P]),
    ("sd_sampler_state", c_int32, [P, c_int32, c_int32, P, c_size_t, c_int64,
                                   ctypes.POINTER(sd_sampler_view)]),
    ("sd_plain_em_workspace", c_size_t, [P, c_int32]),
    ("sd_run_plain_em", c_int32, [P, c_int32, c_uint64, P, P, c_size_t, P]),
    ("sd_latent_attention_workspace", c_size_t, [c_int32] * 5),
    ("sd_latent_attention", c_int32, [c_int32, c_int32, c_int32, c_int32, c_int32, c_int32, c_double, P, SH, P, c_int64,
                                      c_int64, c_int32, c_int32, P, c_int64, c_int32, P, P, P, SH, P, P, c_size_t, P]),
    ("sd_latent_attention_expanded_workspace", c_size_t, [c_int32] * 7),
    ("sd_latent_attention_expanded", c_int32, [c_int32, c_int32, c_int32, c_int32, c_int32, c_int32, c_double, c_int32, P,
                                               SH, c_int32, P, SH, P, c_int64, P, SH, P, P, P, SH, P, P, c_size_t, P]),
    ("sd_token_logprobs_workspace", c_size_t, [c_int32, c_int32, c_int32]),
    ("sd_token_logprobs", c_int32, [c_int32, c_int32, c_int32, P, c_int64, c_double, c_int32, P, P, P, P, c_int32,
                                    P, P, P, c_size_t, P]),
    ("sd_verify_tokens_workspace", c_size_t, [c_int32, c_int32, c_int32]),
    ("sd_verify_tokens", c_int32, [c_int32, c_int32, c_int32, c_int32, c_int32, c_double, P, S, P, S, P, P, P, P,
                                   c_uint64, P, P, P, P, P, P, c_size_t, P]),
    ("sd_latent_append", c_int32, [c_int32] * 7 + [P, P, S, P, S, P, P, P, P, P, c_int64, c_int64, c_int32, c_int32, P,
                                                   c_int64, c_int32, P, S, P, SH, P, SH, P]),
    ("sd_latent_attention_tree_workspace", c_size_t, [c_int32] * 5),
    ("sd_latent_attention_tree", c_int32, [c_int32, c_int32, c_int32, c_int32, c_int32, c_int32, c_double, P, SH, P,
                                           c_int64, c_int64, c_int32, c_int32, P, c_int64, c_int32, P, P, P, P, SH, P, P,
                                           c_size_t, P]),
    ("sd_verify_tree_workspace", c_size_t, [c_int32, c_int32, c_int32]),
    ("sd_verify_tree", c_int32, [c_int32, c_int32, c_int32, c_int32, c_int32, c_double, c_int32, P, S, P, S, P, P, P, P, P,
                                 c_uint64, P, P, P, P, P, c_size_t, P]),
    ("sd_latent_keep", c_int32, [c_int32] * 5 + [P, c_int64, c_int64, c_int64, c_int32, c_int32, P, c_int64, c_int32, P, P,
                                                 P, P, P, P]),
    ("sd_profile_enable", c_int32, [c_int32]),
    ("sd_profile_only", c_int32, [c_char_p]),
    ("sd_profile_every", c_int32, [c_int32]),
    ("sd_profile_seen", c_int32, [c_char_p, ctypes.POINTER(c_int64)]),
    ("sd_profile_read", c_int32, [ctypes.POINTER(sd_kernel_stat), c_int32, ctypes.POINTER(c_int32)]),
    ("sd_philox_words", c_int32, [c_uint64, c_int32, P, P, P]),
    ("sd_philox_normals", c_int32, [c_uint64, c_uint32, c_uint32, c_uint32, c_uint32, c_int32, P, P]),
    ("sd_mfma_loop", c_int32, [c_int32, c_int32, P, P]),
]

_lib = None


def load():
    """Load the library (once).  Raises if it is not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        lib = ctypes.CDLL(LIB_PATH)
        for name, res, args in SIGNATURES:
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def last_error():
    return load().sd_last_error().decode(errors="replace")


def _check(status, name):
    if status != SD_OK:
        raise SpecDiffError(status, f"{name}: {last_error()}")


def _p(t):
    return None if t is None else c_void_p(t.data_ptr())


def _stream():
    import torch
    return c_void_p(torch.cuda.current_stream().cuda_stream)


def stride3(t):
    """sd_stride of a [B][rows][d] view whose last dimension is contiguous."""
    assert t.dim() == 3 and t.stride(2) == 1, "need a [B][rows][d] view with contiguous rows"
    return sd_stride(t.stride(0), t.stride(1))


def schedule(n_steps, beta_min=0.1, beta_max=20.0, churn=1.0):
    return sd_schedule(int(n_steps), float(beta_min), float(beta_max), float(churn))


def sd_abi_version():
    return load().sd_abi_version()


def sd_schedule_table(sched):
    import numpy as np
    out = np.empty((4, sched.n_steps + 1), dtype=np.float64)
    _check(load().sd_schedule_table(ctypes.byref(sched), out.ctypes.data_as(c_void_p)), "sd_schedule_table")
    return out


class Target:
    """Owner of an sd_target handle (Gaussian-mixture target on the current device)."""

    def __init__(self, sched, mu, var, log_w, precision=SD_FP32):
        import numpy as np
        mu = np.ascontiguousarray(mu, dtype=np.float32)
        var = np.ascontiguousarray(var, dtype=np.float32)
        log_w = np.ascontiguousarray(log_w, dtype=np.float32)
        self.sched = sched
        self.M, self.d = mu.shape
        h = c_void_p()
        _check(load().sd_target_create(ctypes.byref(sched), self.d, self.M,
                                       mu.ctypes.data_as(c_void_p), var.ctypes.data_as(c_void_p),
                                       log_w.ctypes.data_as(c_void_p), precision, ctypes.byref(h)),
               "sd_target_create")
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            load().sd_target_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sd_target_mean_workspace(target, rows):
    return load().sd_target_mean_workspace(target.handle, rows)


def sd_target_mean(target, x, step, mq, score=None, ws=None):
    """x, mq, score: [rows][d] float32 (row stride >= d); step: [rows] int32."""
    import torch
    rows = x.shape[0]
    if ws is None:
        ws = torch.empty(sd_target_mean_workspace(target, rows), dtype=torch.uint8, device=x.device)
    _check(load().sd_target_mean(target.handle, rows, _p(x), x.stride(0), _p(step), _p(mq), mq.stride(0),
                                 _p(score), score.stride(0) if score is not None else 0, _p(ws),
                                 ws.numel(), _stream()), "sd_target_mean")


def sd_target_mean_noalloc(target, x, step, mq, score=None):
    """sd_target_mean with the library's own scratch memory (no workspace)."""
    rows = x.shape[0]
    _check(load().sd_target_mean_noalloc(target.handle, rows, _p(x), x.stride(0), _p(step), _p(mq),
                                         mq.stride(0), _p(score),
                                         score.stride(0) if score is not None else 0, _stream()),
           "sd_target_mean_noalloc")


def sd_target_mean_noalloc_max_bytes():
    return load().sd_target_mean_noalloc_max_bytes()


def sd_init_chains(y, seed):
    B, d = y.shape
    _check(load().sd_init_chains(B, d, seed, _p(y), _stream()), "sd_init_chains")


def sd_draft_block(sched, y, cache_score, k, rnd, seed, x, mp):
    """y, cache_score [B][d]; k int32 [B]; rnd int32/uint32 [B]; x [B][K+1][d]; mp [B][K][d] views."""
    B, d = y.shape
    K = mp.shape[1]
    _check(load().sd_draft_block(ctypes.byref(sched), B, K, d, _p(y), _p(cache_score), _p(k), _p(rnd),
                                 seed, _p(x), stride3(x), _p(mp), stride3(mp), _stream()),
           "sd_draft_block")


def _verify_out(B, K, dev):
    import torch
    return dict(tau=torch.empty(B, dtype=torch.int32, device=dev),
                log_alpha_res=torch.empty(B, dtype=torch.float64, device=dev),
                u_res=torch.empty(B, dtype=torch.float64, device=dev),
                delta_norm=torch.empty(B, K, dtype=torch.float64, device=dev),
                log_ratio=torch.empty(B, K, dtype=torch.float64, device=dev),
                coins=torch.empty(B, dtype=torch.int64, device=dev))


def sd_verify_block(y_draft, mp, mq, sigma, kb, rnd, seed, mode=SD_BLOCK, usample_mode=SD_USAMPLE_EXACT,
                    out=None):
    """Views [B][K][d] (mq: [B][>=K][d]); sigma [B][K+1] float64; kb, rnd [B] int32.

    Returns dict of device tensors tau, log_alpha_res, u_res, delta_norm, log_ratio, coins.
    """
    B, K, d = y_draft.shape
    if out is None:
        out = _verify_out(B, K, y_draft.device)
    _check(load().sd_verify_block(B, K, d, mode, _p(y_draft), stride3(y_draft), _p(mp), stride3(mp),
                                  _p(mq), stride3(mq), _p(sigma), _p(kb), _p(rnd), seed, usample_mode,
                                  _p(out["tau"]), _p(out["log_alpha_res"]), _p(out["u_res"]),
                                  _p(out["delta_norm"]), _p(out["log_ratio"]), _p(out.get("coins")),
                                  _stream()), "sd_verify_block")
    return out


def sd_verify_block_tempered(y_draft, mp, mq, sigma, kb, rnd, seed, omega, mode=SD_BLOCK,
                             usample_mode=SD_USAMPLE_EXACT, out=None):
    """sd_verify_block with temperature omega (same arguments and outputs)."""
    B, K, d = y_draft.shape
    if out is None:
        out = _verify_out(B, K, y_draft.device)
    _check(load().sd_verify_block_tempered(B, K, d, mode, float(omega), _p(y_draft), stride3(y_draft),
                                           _p(mp), stride3(mp), _p(mq), stride3(mq), _p(sigma), _p(kb),
                                           _p(rnd), seed, usample_mode, _p(out["tau"]),
                                           _p(out["log_alpha_res"]), _p(out["u_res"]),
                                           _p(out["delta_norm"]), _p(out["log_ratio"]),
                                           _p(out.get("coins")), _stream()), "sd_verify_block_tempered")
    return out


def sd_sample_residual(y_draft, mp, mq, sigma, kb, steps_left, tau, u_res, delta_norm, rnd, seed, y_out):
    B, K, d = y_draft.shape
    _check(load().sd_sample_residual(B, K, d, _p(y_draft), stride3(y_draft), _p(mp), stride3(mp), _p(mq),
                                     stride3(mq), _p(sigma), _p(kb), _p(steps_left), _p(tau), _p(u_res),
                                     _p(delta_norm), _p(rnd), seed, _p(y_out), _stream()),
           "sd_sample_residual")


def sd_sample_residual_reflection(y_draft, mp, mq, sigma, kb, steps_left, tau, rnd, seed, y_out):
    B, K, d = y_draft.shape
    _check(load().sd_sample_residual_reflection(B, K, d, _p(y_draft), stride3(y_draft), _p(mp),
                                                stride3(mp), _p(mq), stride3(mq), _p(sigma), _p(kb),
                                                _p(steps_left), _p(tau), _p(rnd), seed, _p(y_out),
                                                _stream()), "sd_sample_residual_reflection")


def sd_sampler_workspace(target, B, K):
    return load().sd_sampler_workspace(target.handle, B, K)


def _stats_dict(st):
    return dict(rounds=st.rounds, chain_rounds=st.chain_rounds, steps=st.steps, ties=st.ties,
                mean_tau=st.mean_tau, finished=bool(st.finished), groups=st.groups,
                tau_hist=[st.tau_hist[i] for i in range(SD_MAX_BLOCK + 2)])


def sd_run_sampler(target, B, K, seed, mode=SD_BLOCK, usample_mode=SD_USAMPLE_EXACT, y_out=None,
                   trace_rounds=0, ws=None, device="cuda"):
    """Runs Alg. 8 for B chains; returns (y_out [B][d], stats dict, tau_trace or None)."""
    import torch
    if y_out is None:
        y_out = torch.empty(B, target.d, dtype=torch.float32, device=device)
    if ws is None:
        ws = torch.empty(sd_sampler_workspace(target, B, K), dtype=torch.uint8, device=device)
    trace = torch.zeros(trace_rounds, B, dtype=torch.int32, device=device) if trace_rounds > 0 else None
    st = sd_stats()
    _check(load().sd_run_sampler(target.handle, B, K, mode, usample_mode, seed, _p(y_out), _p(trace),
                                 trace_rounds, ctypes.byref(st), _p(ws), ws.numel(), _stream()),
           "sd_run_sampler")
    return y_out, _stats_dict(st), trace


def sd_run_sampler_ex(target, B, K, seed, mode=SD_BLOCK, usample_mode=SD_USAMPLE_EXACT,
                      residual=SD_RESIDUAL_DECOMPOSITION, drafter=SD_DRAFTER_FREE, omega=1.0,
                      y_out=None, trace_rounds=0, ws=None, device="cuda", start_round=0,
                      max_rounds=-1, trace=None, groups=0):
    """Alg. 8 with the sampler options (residual, drafter, temperature, the
    rounds of a run this call does: max_rounds < 0 until done, 0 initialise
    only, and the chain groups run concurrently: 0 the library's choice, 1, 2);
    returns as sd_run_sampler.  A partial run continues with the same ws (and
    trace) and start_round = stats["rounds"]."""
    import torch
    if y_out is None:
        y_out = torch.empty(B, target.d, dtype=torch.float32, device=device)
    if ws is None:
        ws = torch.empty(sd_sampler_workspace(target, B, K), dtype=torch.uint8, device=device)
    if trace is None and trace_rounds > 0:
        trace = torch.zeros(trace_rounds, B, dtype=torch.int32, device=device)
    if trace is not None:
        trace_rounds = trace.shape[0]
    st = sd_stats()
    opts = sd_sampler_options(mode, usample_mode, residual, drafter, float(omega), int(start_round),
                              int(max_rounds), int(groups))
    _check(load().sd_run_sampler_ex(target.handle, B, K, ctypes.byref(opts), seed, _p(y_out), _p(trace),
                                    trace_rounds, ctypes.byref(st), _p(ws), ws.numel(), _stream()),
           "sd_run_sampler_ex")
    return y_out, _stats_dict(st), trace


def sd_sampler_state(target, B, K, ws, rounds):
    """Views (torch tensors aliasing ws) of the sampler state after `rounds` rounds:
    x [B][K+1][d], y [B][d], cache [B][d], cache_step, k, round [B] int32,
    mq [B][K+1][d], lrp [B(K+1)][n_tiles][3] float64, tau [B], coins [B] int64,
    log_alpha_res, u [B] float64, ties [B] int32."""
    import torch
    v = sd_sampler_view()
    _check(load().sd_sampler_state(target.handle, B, K, _p(ws), ws.numel(), int(rounds), ctypes.byref(v)),
           "sd_sampler_state")
    base = ws.data_ptr()
    d, K1 = target.d, K + 1

    def view(ptr, shape, dtype):
        esz = torch.empty((), dtype=dtype).element_size()
        off = ptr - base
        assert off % esz == 0
        n = 1
        for e in shape:
            n *= e
        return ws[off: off + n * esz].view(dtype).view(*shape)

    f32, i32, f64, i64 = torch.float32, torch.int32, torch.float64, torch.int64
    return dict(x=view(v.x, (B, K1, d), f32), y=view(v.y, (B, d), f32), cache=view(v.cache, (B, d), f32),
                cache_step=view(v.cache_step, (B,), i32), k=view(v.k, (B,), i32),
                round=view(v.round, (B,), i32), mq=view(v.mq, (B, K1, d), f32),
                lrp=view(v.lrp, (B * K1, v.n_tiles, 3), f64), tau=view(v.tau, (B,), i32),
                coins=view(v.coins, (B,), i64), log_alpha_res=view(v.log_alpha_res, (B,), f64),
                u=view(v.u, (B,), f64), ties=view(v.ties, (B,), i32))


def sd_plain_em_workspace(target, B):
    return load().sd_plain_em_workspace(target.handle, B)


def sd_run_plain_em(target, B, seed, y_out=None, ws=None, device="cuda"):
    """The plain EM chain for B chains (N target calls); returns Y_N [B][d]."""
    import torch
    if y_out is None:
        y_out = torch.empty(B, target.d, dtype=torch.float32, device=device)
    if ws is None:
        ws = torch.empty(sd_plain_em_workspace(target, B), dtype=torch.uint8, device=device)
    _check(load().sd_run_plain_em(target.handle, B, seed, _p(y_out), _p(ws), ws.numel(), _stream()),
           "sd_run_plain_em")
    return y_out


_types = {}


def _type(t):
    if not _types:
        import torch
        _types.update({torch.float32: SD_TYPE_F32, torch.bfloat16: SD_TYPE_BF16, torch.float16: SD_TYPE_F16})
    if t.dtype not in _types:
        raise SpecDiffError(SD_EINVAL, f"unsupported element type {t.dtype}")
    return _types[t.dtype]


def _need(cond, name, what):
    if not cond:
        raise SpecDiffError(SD_EINVAL, f"{name}: {what}")


def _operands(name, types, **tensors):
    """Refuses operands that are not on the current device, or not of the type that `types` states.

    Returns the current stream's handle."""
    import torch
    dev = torch.cuda.current_device() if next(iter(tensors.values())).is_cuda else 0
    for what, t in tensors.items():
        if t is not None and t.get_device() != dev:  # (-1: in the host's memory)
            _need(False, name, f"{what} is on {t.device}, not on the current GPU")
    for what, want in types.items():
        t = tensors[what]
        if t is not None and t.dtype != want:
            _need(False, name, f"{what} must be {want}, not {t.dtype}")
    ws = tensors.get("ws")
    _need(ws is None or ws.is_contiguous(), name, "ws must be contiguous")
    return torch._C._cuda_getCurrentRawStream(dev)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _workspace(need, device):
    import torch
    return torch.empty(need, dtype=torch.uint8, device=device)


def sd_latent_attention_workspace(B, Q, H, d_latent, d_rope):
    return load().sd_latent_attention_workspace(B, Q, H, d_latent, d_rope)


def sd_latent_attention(q, cache, lens, d_latent, pages=None, rows=None, scale=None, out=None, lse=None, ws=None):
    """q [B][Q][H][d_latent + d_rope] and cache [n_pages][page_size][d_latent + d_rope] of one
    16-bit type (last dimension contiguous); lens [B], pages [B][max_pages] (None: page b is
    sequence b), rows [B] (None: Q rows each) int32.

    scale: a model's absorbed scores are those of its expanded form, whose scale is
    (d_nope + d_rope)^-1/2 of the heads' own width d_nope; that cannot be read off the operands.
    Without one (d_latent + d_rope)^-1/2 is taken, with a warning: attention to the cached
    vectors for their own sake.

    Returns (out [B][Q][H][d_latent], lse [B][Q][H] float32).
    """
    return _attention("sd_latent_attention", q, cache, lens, None, d_latent, pages, rows, scale, out, lse, ws)


def _attention(name, q, cache, lens, parents, d_latent, pages, rows, scale, out, lse, ws):
    import torch
    i32, tree = torch.int32, parents is not None
    if scale is None:
        warnings.warn(f"{name}: no scale given, (d_latent + d_rope)^-1/2 is taken; a model's absorbed attention has "
                      "(d_nope + d_rope)^-1/2", stacklevel=3)
    _need(q.dim() == 4 and cache.dim() == 3 and q.stride(3) == 1 and cache.stride(2) == 1, name,
          "q must be [B][Q][H][d] and cache [n_pages][page_size][d] with contiguous d")
    B, Q, H, d = q.shape
    _need(cache.shape[2] == d and cache.dtype == q.dtype, name, "q and cache must agree in d and type")
    _need(0 < d_latent <= d, name, f"d_latent = {d_latent} is not in [1, {d}]")
    if out is None:
        out = torch.empty(B, Q, H, d_latent, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(B, Q, H, dtype=torch.float32, device=q.device)
    stream = _operands(name, dict(lens=i32, pages=i32, rows=i32, out=q.dtype, lse=torch.float32, ws=torch.uint8,
                                  parents=i32),
                       q=q, cache=cache, lens=lens, pages=pages, rows=rows, out=out, lse=lse, ws=ws, parents=parents)
    _need(lens.shape == (B,) and lens.is_contiguous(), name, "lens must be contiguous [B]")
    _need(not tree or (parents.shape == (B, Q) and parents.is_contiguous()), name, "parents must be contiguous [B][Q]")
    _need(rows is None or (rows.shape == (B,) and rows.is_contiguous()), name, "rows must be contiguous [B]")
    _need(pages is None or (pages.dim() == 2 and pages.shape[0] == B and pages.stride(1) == 1), name,
          "pages must be [B][max_pages] with contiguous rows")
    _need(out.shape == (B, Q, H, d_latent) and out.stride(3) == 1, name, "out must be [B][Q][H][d_latent]")
    _need(lse.shape == (B, Q, H) and lse.is_contiguous(), name, "lse must be contiguous [B][Q][H]")
    lib = load()
    size, call = (lib.sd_latent_attention_tree_workspace, lib.sd_latent_attention_tree) if tree else \
        (lib.sd_latent_attention_workspace, lib.sd_latent_attention)
    if ws is None:
        ws = _workspace(size(B, Q, H, d_latent, d - d_latent), q.device)
    _check(call(B, Q, H, d_latent, d - d_latent, _type(q), d ** -0.5 if scale is None else float(scale), q.data_ptr(),
                sd_stride_h(*q.stride()[:3]), cache.data_ptr(), cache.stride(0), cache.stride(1), cache.shape[0],
                cache.shape[1], _ptr(pages), 0 if pages is None else pages.stride(0),
                0 if pages is None else pages.shape[1], lens.data_ptr(), _ptr(rows),
                *((parents.data_ptr(),) if tree else ()), out.data_ptr(), sd_stride_h(*out.stride()[:3]),
                lse.data_ptr(), ws.data_ptr(), ws.numel(), stream), name)
    return out, lse


def sd_latent_attention_expanded_workspace(n, H, d_nope, d_rope, d_v, Tq, Tk):
    return load().sd_latent_attention_expanded_workspace(n, H, d_nope, d_rope, d_v, Tq, Tk)


def sd_latent_attention_expanded(q, k, k_rope, v, cu_q, cu_k, scale=None, out=None, lse=None, ws=None):
    """q [Tq][H][d_nope + d_rope], k [Tk][H][d_nope], k_rope [Tk][d_rope] (None: d_rope = 0), v [Tk][H][d_v]
    of one 16-bit type (last dimension contiguous); cu_q, cu_k [n+1] int32 offsets of the sequences;
    scale defaults to (d_nope + d_rope)^-1/2.

    Returns (out [Tq][H][d_v], lse [Tq][H] float32).
    """
    import torch
    name, i32 = "sd_latent_attention_expanded", torch.int32
    _need(q.dim() == 3 and k.dim() == 3 and v.dim() == 3 and q.stride(2) == k.stride(2) == v.stride(2) == 1, name,
          "q, k and v must be [tokens][H][d] with contiguous d")
    Tq, H, d = q.shape
    Tk, _, dn = k.shape
    dr, dv = d - dn, v.shape[2]
    _need(dn > 0, name, "d_nope = 0")
    _need(k.shape[1] == H and tuple(v.shape[:2]) == (Tk, H) and k.dtype == v.dtype == q.dtype, name,
          "q, k and v must agree in heads, tokens and type")
    _need((k_rope is None and dr == 0) or (k_rope is not None and tuple(k_rope.shape) == (Tk, dr) and
                                           k_rope.dtype == q.dtype and k_rope.stride(1) == 1), name,
          "k_rope must be [Tk][d_rope] of q's type with contiguous rows")
    if out is None:
        out = torch.empty(Tq, H, dv, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(Tq, H, dtype=torch.float32, device=q.device)
    stream = _operands(name, dict(cu_q=i32, cu_k=i32, out=q.dtype, lse=torch.float32, ws=torch.uint8),
                       q=q, k=k, k_rope=k_rope, v=v, cu_q=cu_q, cu_k=cu_k, out=out, lse=lse, ws=ws)
    n = cu_q.numel() - 1
    _need(cu_q.dim() == 1 and cu_k.shape == (n + 1,) and cu_q.is_contiguous() and cu_k.is_contiguous(), name,
          "cu_q and cu_k must be contiguous [n + 1]")
    _need(out.shape == (Tq, H, dv) and out.stride(2) == 1, name, "out must be [Tq][H][d_v]")
    _need(lse.shape == (Tq, H) and lse.is_contiguous(), name, "lse must be contiguous [Tq][H]")
    if ws is None:
        need = sd_latent_attention_expanded_workspace(n, H, dn, dr, dv, Tq, Tk)
        ws = _workspace(need, q.device) if need > 0 else None
    strides = [sd_stride_h(0, *x.stride()[:2]) for x in (q, k, v, out)]
    _check(load().sd_latent_attention_expanded(n, H, dn, dr, dv, _type(q), d ** -0.5 if scale is None else float(scale),
                                               Tq, q.data_ptr(), strides[0], Tk, k.data_ptr(), strides[1], _ptr(k_rope),
                                               k_rope.stride(0) if k_rope is not None else 0, v.data_ptr(), strides[2],
                                               cu_q.data_ptr(), cu_k.data_ptr(), out.data_ptr(), strides[3],
                                               lse.data_ptr(), _ptr(ws), ws.numel() if ws is not None else 0, stream), name)
    return out, lse


def sd_token_logprobs_workspace(rows, V, n_top=0):
    return load().sd_token_logprobs_workspace(rows, V, n_top)


def sd_token_logprobs(logits, tokens=None, n_top=0, temperature=1.0, ws=None):
    """logits [rows][V] (float32, bfloat16 or float16; rows contiguous); tokens [rows] or [rows][n_tok] int32.

    Returns dict of device tensors lse, entropy [rows] and, where asked for, logprob (as
    tokens) and top_ids, top_logprobs [rows][n_top].
    """
    import torch
    name, i32 = "sd_token_logprobs", torch.int32
    _need(logits.dim() == 2 and (logits.stride(1) == 1 or logits.shape[1] == 1), name, "logits must be [rows][V] with contiguous rows")
    rows, V = logits.shape
    stream = _operands(name, dict(tokens=i32, ws=torch.uint8), logits=logits, tokens=tokens, ws=ws)
    n_tok = 0
    if tokens is not None:
        _need(tokens.dim() in (1, 2) and tokens.shape[0] == rows and tokens.is_contiguous(), name,
              "tokens must be contiguous [rows] or [rows][n_tok]")
        n_tok = 1 if tokens.dim() == 1 else tokens.shape[1]
    f32, dev = torch.float32, logits.device
    lse, entropy = torch.empty(rows, dtype=f32, device=dev), torch.empty(rows, dtype=f32, device=dev)
    logprob = ids = tops = None
    out = dict(lse=lse, entropy=entropy)
    if tokens is not None:
        out["logprob"] = logprob = torch.empty(tokens.shape, dtype=f32, device=dev)
    if n_top > 0:
        out["top_ids"] = ids = torch.empty(rows, n_top, dtype=i32, device=dev)
        out["top_logprobs"] = tops = torch.empty(rows, n_top, dtype=f32, device=dev)
    if ws is None:
        ws = _workspace(sd_token_logprobs_workspace(rows, V, n_top), dev)
    _check(load().sd_token_logprobs(rows, V, _type(logits), logits.data_ptr(), logits.stride(0) if rows > 1 else V,
                                    float(temperature), n_tok, _ptr(tokens), _ptr(logprob), entropy.data_ptr(),
                                    lse.data_ptr(), n_top, _ptr(ids), _ptr(tops), ws.data_ptr(), ws.numel(), stream), name)
    return out


def sd_verify_tokens_workspace(B, K, V):
    return load().sd_verify_tokens_workspace(B, K, V)


def sd_verify_tokens(draft, target, tokens, kb, uniforms=None, rnd=None, seed=0, mode=SD_BLOCK, temperature=1.0,
                     ws=None, out=None):
    """draft [B][K][V], target [B][K+1][V] logits of one type (rows contiguous); tokens [B][K],
    kb [B] int32; uniforms [B][K+1] float64, or rnd [B] int32/uint32 and the seed.

    Returns dict of device tensors tau, token [B] int32, log_alpha_res [B], log_ratio [B][K]
    float32, coins [B] int64.
    """
    import torch
    name, i32, f32 = "sd_verify_tokens", torch.int32, torch.float32
    _need(draft.dim() == 3 and target.dim() == 3, name, "draft and target must be [B][K][V] and [B][K+1][V]")
    B, K, V = draft.shape
    _need(target.shape == (B, K + 1, V), name, "target must be [B][K+1][V]")
    _need(draft.dtype == target.dtype, name, "draft and target must be of one type")
    stream = _operands(name, dict(tokens=i32, kb=i32, uniforms=torch.float64, ws=torch.uint8),
                       draft=draft, target=target, tokens=tokens, kb=kb, uniforms=uniforms, rnd=rnd, ws=ws)
    _need(tokens.shape == (B, K) and tokens.is_contiguous(), name, "tokens must be contiguous [B][K]")
    _need(kb.shape == (B,) and kb.is_contiguous(), name, "kb must be contiguous [B]")
    _need(uniforms is None or (uniforms.shape == (B, K + 1) and uniforms.is_contiguous()), name,
          "uniforms must be contiguous [B][K+1]")
    _need(rnd is None or (rnd.shape == (B,) and rnd.dtype in (torch.int32, torch.uint32) and rnd.is_contiguous()), name,
          "rnd must be contiguous [B] of int32 or uint32")
    if out is None:
        dev = draft.device
        out = dict(tau=torch.empty(B, dtype=i32, device=dev), token=torch.empty(B, dtype=i32, device=dev),
                   log_alpha_res=torch.empty(B, dtype=f32, device=dev), log_ratio=torch.empty(B, K, dtype=f32, device=dev),
                   coins=torch.empty(B, dtype=torch.int64, device=dev))
    else:
        said = dict(tau=i32, token=i32, log_alpha_res=f32, log_ratio=f32, coins=torch.int64)
        _need(all(out.get(k) is not None for k in said if k != "coins"), name,
              "out must hold tau, token, log_alpha_res and log_ratio")
        _operands(name, said, **{k: out.get(k) for k in said})
        for k in said:
            o = out.get(k)
            _need(o is None or (o.shape == ((B, K) if k == "log_ratio" else (B,)) and o.is_contiguous()), name,
                  f"{k} must be contiguous [B][K]" if k == "log_ratio" else f"{k} must be contiguous [B]")
    if ws is None:
        ws = _workspace(sd_verify_tokens_workspace(B, K, V), draft.device)
    _check(load().sd_verify_tokens(B, K, V, mode, _type(draft), float(temperature), draft.data_ptr(), stride3(draft),
                                   target.data_ptr(), stride3(target), tokens.data_ptr(), kb.data_ptr(), _ptr(uniforms),
                                   _ptr(rnd), seed, out["tau"].data_ptr(), out["token"].data_ptr(),
                                   out["log_alpha_res"].data_ptr(), out["log_ratio"].data_ptr(), _ptr(out.get("coins")),
                                   ws.data_ptr(), ws.numel(), stream), name)
    return out


def _table(name, pages, B):
    """Width and row stride of a page table."""
    if pages is None:
        return 0, 0
    shape, stride = pages.shape, pages.stride()
    _need(len(shape) == 2 and shape[0] == B and stride[1] == 1, name, "pages must be [B][max_pages] with contiguous rows")
    return shape[1], stride[0]


def sd_latent_append(latent, k_rope, cache, lens, freq, pages=None, rows=None, cu=None, parents=None, q=None, q_out=None,
                     k_out=None, rope=SD_ROPE_PAIRS):
    """latent [B][Q][d_latent], k_rope [B][Q][d_rope] (None: d_rope = 0) into cache [n_pages][page_size][d_latent +
    d_rope], all of one 16-bit type (last dimension contiguous); lens [B], rows [B] (None: Q each), parents [B][Q] (None:
    a chain), pages [B][max_pages] (None: page b is sequence b) int32; freq [d_rope / 2] float64.  With cu [B + 1]
    int32 the rows are ragged: [T][..] in the place of [B][Q][..].
    q [B][Q][H][d_rope]: turned by the rows' positions too, into q_out (None: a new tensor; q: in place).
    k_out [B][Q][d_rope] (k_rope: in place): the turned k_rope once more.

    Returns q_out (None without q).
    """
    import torch
    name, i32, f64 = "sd_latent_append", torch.int32, torch.float64
    # (shapes and strides are read once: each reading is as long as several comparisons)
    lead, ls, cs = 1 if cu is not None else 2, latent.shape, cache.shape
    lst, cst = latent.stride(), cache.stride()
    _need(len(ls) == lead + 1 and len(cs) == 3 and lst[lead] == 1 and cst[2] == 1, name,
          "latent must be [B][Q][d_latent], or [T][d_latent] with cu, and cache [n_pages][page_size][d] with contiguous d")
    dc, t, tokens = ls[lead], latent.dtype, ls[:lead]
    dr, H, none = cs[2] - dc, 0, sd_stride_h(0, 0, 0)
    kst = None if k_rope is None else k_rope.stride()
    _need((k_rope is None and dr == 0) or (k_rope is not None and k_rope.shape == (*tokens, dr) and kst[lead] == 1), name,
          "k_rope must be as latent with the rest of the cache's d, contiguous")
    _need(q is not None or q_out is None, name, "q_out goes with q")
    qst = ost = none
    if q is not None:
        qs, qst = q.shape, q.stride()
        _need(len(qs) == lead + 2 and qs[:lead] == tokens and qs[lead + 1] == dr and qst[lead + 1] == 1 and qs[lead] > 0, name,
              "q must be [B][Q][H][d_rope], or [T][H][d_rope] with cu, contiguous in d")
        H = qs[lead]
        if q_out is None:
            q_out = torch.empty(qs, dtype=q.dtype, device=q.device)
        ost = q_out.stride()
        _need(q_out.shape == qs and ost[lead + 1] == 1, name, "q_out must be as q, contiguous in d")
        qst = sd_stride_h(0, qst[0], qst[1]) if lead == 1 else sd_stride_h(qst[0], qst[1], qst[2])
        ost = sd_stride_h(0, ost[0], ost[1]) if lead == 1 else sd_stride_h(ost[0], ost[1], ost[2])
    ko = None if k_out is None else k_out.stride()
    _need(k_out is None or (k_rope is not None and k_out.shape == k_rope.shape and ko[lead] == 1), name,
          "k_out must be as k_rope, contiguous in d")
    stream = _operands(name, dict(k_rope=t, cache=t, q=t, q_out=t, k_out=t, lens=i32, freq=f64, pages=i32, rows=i32, cu=i32,
                                  parents=i32),
                       latent=latent, k_rope=k_rope, cache=cache, lens=lens, freq=freq, pages=pages, rows=rows, cu=cu,
                       parents=parents, q=q, q_out=q_out, k_out=k_out)
    _need(lens.dim() == 1 and lens.is_contiguous(), name, "lens must be contiguous [B]")
    B, Q = lens.shape[0], ls[lead - 1]
    _need(cu is not None or ls[0] == B, name, "latent and lens must agree in B")
    _need(cu is None or (cu.shape == (B + 1,) and cu.is_contiguous()), name, "cu must be contiguous [B + 1]")
    _need(dr == 0 or (freq is not None and freq.shape == (dr // 2,) and freq.is_contiguous()), name,
          "freq must be contiguous [d_rope / 2]")
    _need(rows is None or (rows.shape == (B,) and rows.is_contiguous()), name, "rows must be contiguous [B]")
    _need(parents is None or (parents.shape == (B, Q) and parents.is_contiguous()), name, "parents must be contiguous [B][Q]")
    width, pst = _table(name, pages, B)

    def stride(x):
        return sd_stride(0, 0) if x is None else sd_stride(0, x[0]) if lead == 1 else sd_stride(x[0], x[1])

    _check(load().sd_latent_append(B, Q, H, dc, dr, _type(latent), rope, _ptr(freq), latent.data_ptr(), stride(lst),
                                   _ptr(k_rope), stride(kst), _ptr(cu), _ptr(parents), lens.data_ptr(), _ptr(rows),
                                   cache.data_ptr(), cst[0], cst[1], cs[0], cs[1], _ptr(pages), pst, width, _ptr(k_out),
                                   stride(ko), _ptr(q), qst, _ptr(q_out), ost, stream), name)
    return q_out


def sd_latent_attention_tree_workspace(B, Q, H, d_latent, d_rope):
    return load().sd_latent_attention_tree_workspace(B, Q, H, d_latent, d_rope)


def sd_latent_attention_tree(q, cache, lens, parents, d_latent, pages=None, rows=None, scale=None, out=None, lse=None,
                             ws=None):
    """sd_latent_attention where row i sees the prefix, itself and its ancestors: parents [B][Q] int32, an
    earlier node's number (any other value: none)."""
    _need(parents is not None, "sd_latent_attention_tree", "parents must be contiguous [B][Q]")
    return _attention("sd_latent_attention_tree", q, cache, lens, parents, d_latent, pages, rows, scale, out, lse, ws)


def sd_verify_tree_workspace(B, Q, V):
    return load().sd_verify_tree_workspace(B, Q, V)


def sd_verify_tree(draft, target, tokens, parents, rows=None, draws=SD_TREE_IID, max_children=None, uniforms=None, rnd=None,
                   seed=0, temperature=1.0, ws=None, out=None):
    """draft (None with SD_TREE_GIVEN) and target [B][Q][V] logits of one type (rows contiguous); tokens, parents
    [B][Q], rows [B] (None: Q each) int32; uniforms [B][Q] float64, or rnd [B] int32/uint32 and the seed.
    max_children: how many children of a node are tried at most (None, Q or more: all).  Each one more is one more kernel but with
    SD_TREE_GIVEN, whether a node has so many or not: a caller says what its trees have (trees of 64 nodes with up to 4
    children, independent draws, 4 / None: one over 32000 tokens 40 / 254 us, 32 over 131072 197 / 479 us).

    Returns dict of device tensors tau, token [B], path [B][Q] int32, accept [B][Q] float32.
    """
    import torch
    name, i32, f32 = "sd_verify_tree", torch.int32, torch.float32
    shape, tst = target.shape, target.stride()
    _need(len(shape) == 3, name, "target must be [B][Q][V]")
    B, Q, V = shape
    _need(draft is None or (draft.shape == shape and draft.dtype == target.dtype), name,
          "draft and target must be [B][Q][V] of one type")
    dst = tst if draft is None else draft.stride()
    _need(tst[2] == 1 and dst[2] == 1, name, "draft and target must have contiguous rows")
    stream = _operands(name, dict(tokens=i32, parents=i32, rows=i32, uniforms=torch.float64, ws=torch.uint8),
                       target=target, draft=draft, tokens=tokens, parents=parents, rows=rows, uniforms=uniforms, rnd=rnd,
                       ws=ws)
    for what, x in (("tokens", tokens), ("parents", parents), ("uniforms", uniforms)):
        if x is not None and not (x.shape == (B, Q) and x.is_contiguous()):
            _need(False, name, f"{what} must be contiguous [B][Q]")
    _need(rows is None or (rows.shape == (B,) and rows.is_contiguous()), name, "rows must be contiguous [B]")
    _need(rnd is None or (rnd.shape == (B,) and rnd.dtype in (torch.int32, torch.uint32) and rnd.is_contiguous()), name,
          "rnd must be contiguous [B] of int32 or uint32")
    if out is None:
        dev = target.device
        out = dict(tau=torch.empty(B, dtype=i32, device=dev), token=torch.empty(B, dtype=i32, device=dev),
                   path=torch.empty(B, Q, dtype=i32, device=dev), accept=torch.empty(B, Q, dtype=f32, device=dev))
    else:
        said = dict(tau=i32, token=i32, path=i32, accept=f32)
        _need(all(out.get(k) is not None for k in said if k != "accept"), name, "out must hold tau, token and path")
        _operands(name, said, **{k: out.get(k) for k in said})
        for k in said:
            o, wide = out.get(k), k in ("path", "accept")
            _need(o is None or (o.shape == ((B, Q) if wide else (B,)) and o.is_contiguous()), name,
                  f"{k} must be contiguous {'[B][Q]' if wide else '[B]'}")
    if ws is None:
        ws = _workspace(sd_verify_tree_workspace(B, Q, V), target.device)
    _check(load().sd_verify_tree(B, Q, V, draws, _type(target), float(temperature), Q if max_children is None else min(max_children, Q),
                                 _ptr(draft), sd_stride(dst[0], dst[1]), target.data_ptr(),
                                 sd_stride(tst[0], tst[1]), tokens.data_ptr(), parents.data_ptr(), _ptr(rows), _ptr(uniforms),
                                 _ptr(rnd), seed, out["tau"].data_ptr(), out["token"].data_ptr(), out["path"].data_ptr(),
                                 _ptr(out.get("accept")), ws.data_ptr(), ws.numel(), stream), name)
    return out


def sd_latent_keep(cache, lens, tau, path, pages=None, rows=None, new_lens=None):
    """cache [n_pages][page_size][d] or [layers][n_pages][page_size][d] of a 16-bit type (d contiguous); lens, tau [B],
    path [B][Q] (sd_verify_tree's), rows [B] (None: Q each), pages [B][max_pages] (None: page b is sequence b) int32.

    Returns new_lens [B] int32 (None: a new tensor; none of lens, rows, tau or path).
    """
    import torch
    name, i32 = "sd_latent_keep", torch.int32
    shape, strides = cache.shape, cache.stride()
    _need(len(shape) in (3, 4) and strides[-1] == 1, name, "cache must be [layers][n_pages][page_size][d] with contiguous d")
    _need(path.dim() == 2 and path.is_contiguous(), name, "path must be contiguous [B][Q]")
    B, Q = path.shape
    if new_lens is None:
        new_lens = torch.empty(B, dtype=i32, device=cache.device)
    stream = _operands(name, dict(lens=i32, tau=i32, path=i32, pages=i32, rows=i32, new_lens=i32),
                       cache=cache, lens=lens, tau=tau, path=path, pages=pages, rows=rows, new_lens=new_lens)
    for what, x in (("lens", lens), ("tau", tau), ("rows", rows), ("new_lens", new_lens)):
        if x is not None and not (x.shape == (B,) and x.is_contiguous()):
            _need(False, name, f"{what} must be contiguous [B]")
    width, pst = _table(name, pages, B)
    layers, layer = (shape[0], strides[0]) if len(shape) == 4 else (1, 0)
    _check(load().sd_latent_keep(layers, B, Q, shape[-1], _type(cache), cache.data_ptr(), layer, strides[-3], strides[-2],
                                 shape[-3], shape[-2], _ptr(pages), pst, width, lens.data_ptr(), _ptr(rows), tau.data_ptr(),
                                 path.data_ptr(), new_lens.data_ptr(), stream), name)
    return new_lens


def sd_profile_enable(on=True):
    _check(load().sd_profile_enable(1 if on else 0), "sd_profile_enable")


def sd_profile_only(name=None):
    _check(load().sd_profile_only(None if name is None else name.encode()), "sd_profile_only")


def sd_profile_every(n):
    _check(load().sd_profile_every(int(n)), "sd_profile_every")


def sd_profile_seen(name):
    n = c_int64()
    _check(load().sd_profile_seen(name.encode(), ctypes.byref(n)), "sd_profile_seen")
    return n.value


def sd_profile_read():
    cap = 64
    arr = (sd_kernel_stat * cap)()
    n = c_int32()
    _check(load().sd_profile_read(arr, cap, ctypes.byref(n)), "sd_profile_read")
    return {arr[i].name.decode(): (arr[i].launches, arr[i].total_ms) for i in range(min(n.value, cap))}


def sd_philox_words(seed, counters, out):
    _check(load().sd_philox_words(seed, counters.shape[0], _p(counters), _p(out), _stream()),
           "sd_philox_words")


def sd_philox_normals(seed, chain, rnd, tag, slot, out):
    _check(load().sd_philox_normals(seed, chain, rnd, tag, slot, out.numel(), _p(out), _stream()),
           "sd_philox_normals")


def sd_mfma_loop(blocks, iters, out):
    """Matrix-core calibration loop: blocks x 16 x iters x 32768 bf16 flops; out [blocks][4] float32."""
    _check(load().sd_mfma_loop(blocks, iters, _p(out), _stream()), "sd_mfma_loop")
