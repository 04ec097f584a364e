"""Thin ctypes binding of the C ABI declared in ``include/rsd.h``.

Argument marshalling only: every function here forwards to the entry point of
the same name in ``librsd.so``.  Device buffers are torch tensors (torch is
used for device memory and the stream handle, nothing else); host buffers are
NumPy arrays.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

__all__ = ["RSD_OK", "RSD_EINVAL", "RSD_ENOMEM", "RSD_ESTATE", "RSD_EHIP", "RSD_DRAFT", "RSD_TARGET", "RSD_PRM",
           "RsdError", "Context", "load_library", "rsd_init", "rsd_set_prompts", "rsd_set_uniforms",
           "rsd_set_criterion", "rsd_step", "rsd_generate", "rsd_export_state", "rsd_export_pages",
           "rsd_set_teacher", "rsd_export_sampled", "rsd_forward", "rsd_sample", "rsd_stage_ms", "rsd_decode_stats", "rsd_destroy",
           "rsd_probe_start", "rsd_probe_read", "rsd_probe_clock", "rsd_iter_stats", "rsd_iter_rows", "rsd_check_rows", "rsd_debug_build", "rsd_probe_attention", "rsd_sample_static",
           "rsd_bon_step", "rsd_bon_generate", "rsd_bon_stats", "EXPORTED_SYMBOLS"]

RSD_OK, RSD_EINVAL, RSD_ENOMEM, RSD_ESTATE, RSD_EHIP = 0, -1, -2, -3, -4
RSD_DRAFT, RSD_TARGET, RSD_PRM = 0, 1, 2
RSD_MERGE_NONE, RSD_MERGE_DRAFT, RSD_MERGE_TARGET = 0, 1, 2
EXPORTED_SYMBOLS = ["rsd_init", "rsd_set_prompts", "rsd_set_uniforms", "rsd_set_criterion", "rsd_step",
                    "rsd_generate", "rsd_export_state", "rsd_export_pages", "rsd_set_teacher",
                    "rsd_export_sampled", "rsd_set_teacher_sd", "rsd_export_proposed", "rsd_set_uniforms_sd", "rsd_sd_verify", "rsd_forward", "rsd_sample", "rsd_stage_ms", "rsd_decode_stats", "rsd_probe_start", "rsd_probe_read", "rsd_probe_clock",
                    "rsd_iter_stats", "rsd_iter_rows", "rsd_check_rows", "rsd_debug_build", "rsd_probe_attention", "rsd_sample_static", "rsd_bon_step", "rsd_bon_generate", "rsd_bon_stats",
                    "rsd_last_error", "rsd_destroy"]
LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librsd.so")


class RsdError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"rsd error {code}: {text}")
        self.code = code


class _Shape(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("rope_theta", C.c_float), ("rms_eps", C.c_float),
                ("dtype", C.c_int32), ("head_kind", C.c_int32)]


class _Weights(C.Structure):
    _fields_ = [("blob", C.c_void_p), ("nbytes", C.c_uint64)]


class _Params(C.Structure):
    _fields_ = [("delta", C.c_float), ("omega_kind", C.c_int32), ("omega_a", C.c_float), ("sep_id", C.c_int32),
                ("eos_id", C.c_int32), ("step_cap", C.c_int32), ("max_steps", C.c_int32), ("max_ctx", C.c_int32),
                ("temperature", C.c_float), ("top_p", C.c_float), ("sep_logit_bias", C.c_float),
                ("page_tokens", C.c_int32), ("kv_pool_bytes", C.c_uint64 * 3), ("use_graphs", C.c_int32),
                ("merge_prm", C.c_int32), ("sd_k", C.c_int32), ("bon_n", C.c_int32)]


class _StepOut(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("draft_len", "draft_tokens", "reward", "accepted", "own_accept",
                                          "final_len", "final_tokens", "finished", "sd_rounds", "sd_proposed",
                                          "sd_kept")]


class _BonOut(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("cand_len", "cand_tokens", "cand_reward", "chosen", "own_choice", "finished",
                                          "ctx_len", "kv_len", "n_pages")]


class _GenOut(C.Structure):
    _fields_ = [("tokens", C.c_void_p), ("ctx_len", C.c_void_p), ("finished", C.c_void_p), ("steps_run", C.c_int32),
                ("n_committed", C.c_int64), ("n_draft", C.c_int64), ("n_target", C.c_int64),
                ("n_accept", C.c_int64), ("n_reject", C.c_int64), ("n_sd_rounds", C.c_int64),
                ("n_sd_proposed", C.c_int64), ("n_sd_kept", C.c_int64)]


_lib = None


def load_library(path: Optional[str] = None):
    """Load ``librsd.so``; raises if it has not been built."""
    global _lib
    if _lib is None or path is not None:
        p = path or LIB_PATH
        if not os.path.exists(p):
            raise RuntimeError(f"{p} is missing: build it first (python -m paper_2501_19324_amd.build); "
                               "there is no fallback path")
        lib = C.CDLL(p)
        lib.rsd_last_error.restype = C.c_char_p
        lib.rsd_last_error.argtypes = [C.c_void_p]
        lib.rsd_destroy.restype = None
        lib.rsd_destroy.argtypes = [C.c_void_p]
        _lib = lib
    return _lib


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _dev_ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous()
    return C.c_void_p(t.data_ptr())


class Context:
    """Owner of one ``rsd_ctx``.  Keeps references to every borrowed buffer."""

    def __init__(self):
        self.handle = C.c_void_p()
        self.keep = {}
        self.batch = 0
        self.max_ctx = 0
        self.step_cap = 0
        self.max_steps = 0
        self.vocab = 0
        self.sd_k = 0

    def check(self, rc: int):
        if rc != RSD_OK:
            raise RsdError(rc, load_library().rsd_last_error(self.handle).decode())

    def __del__(self):
        try:
            rsd_destroy(self)
        except Exception:
            pass


def _shape_struct(s) -> _Shape:
    dtype = {"f32": 0, "bf16": 1}[s.dtype] if isinstance(s.dtype, str) else int(s.dtype)
    head = {"lm": 0, "reward": 1}[s.head_kind] if isinstance(s.head_kind, str) else int(s.head_kind)
    return _Shape(s.n_layers, s.d_model, s.n_heads, s.n_kv_heads, s.d_ffn, s.vocab, s.rope_theta, s.rms_eps, dtype, head)


def rsd_init(shapes: Sequence, weights: Sequence, *, batch: int, delta: float, sep_id: int, step_cap: int,
             max_steps: int, max_ctx: int, eos_id: int = -1, temperature: float = 0.0, top_p: float = 1.0,
             sep_logit_bias: float = 0.0, omega_kind: int = 0, omega_a: float = 0.0, page_tokens: int = 16,
             kv_pool_bytes=(0, 0, 0), use_graphs: int = 1, merge_prm: int = 0, sd_k: int = 0, bon_n: int = 0,
             stream=None) -> Context:
    """``weights``: three device tensors holding each model's blob (with ``merge_prm`` the third holds
    only the reward projection ``w_r`` and ``b_r``; with ``bon_n`` the second may be ``None``)."""
    import torch

    lib = load_library()
    ctx = Context()
    sh = (_Shape * 3)(*[_shape_struct(s) for s in shapes])
    ws = (_Weights * 3)(*[_Weights(None, 0) if w is None else _Weights(w.data_ptr(), w.numel() * w.element_size()) for w in weights])
    p = _Params(delta, omega_kind, omega_a, sep_id, eos_id, step_cap, max_steps, max_ctx, temperature, top_p,
                sep_logit_bias, page_tokens, (C.c_uint64 * 3)(*[int(x) for x in kv_pool_bytes]), use_graphs, merge_prm, sd_k, bon_n)
    st = stream if stream is not None else torch.cuda.current_stream()
    ctx.keep["weights"] = list(weights)
    ctx.keep["stream"] = st
    ctx.batch, ctx.max_ctx, ctx.step_cap, ctx.max_steps, ctx.vocab = batch, max_ctx, step_cap, max_steps, shapes[0].vocab
    ctx.shapes = list(shapes)
    ctx.sd_k = sd_k
    ctx.bon_n = bon_n
    ctx.n_seq = batch // bon_n if bon_n else batch
    rc = lib.rsd_init(C.byref(ctx.handle), sh, ws, C.byref(p), C.c_int32(batch), C.c_void_p(st.cuda_stream))
    ctx.check(rc)
    return ctx


def rsd_destroy(ctx: Context) -> None:
    if ctx.handle:
        load_library().rsd_destroy(ctx.handle)
        ctx.handle = C.c_void_p()
        ctx.keep.clear()


def rsd_set_prompts(ctx: Context, tokens_dev, prompt_len: np.ndarray) -> None:
    pl = np.ascontiguousarray(prompt_len, dtype=np.int32)
    assert tuple(tokens_dev.shape) == (ctx.n_seq, ctx.max_ctx) and tokens_dev.dtype.itemsize == 4 and pl.shape == (ctx.n_seq,)
    ctx.check(load_library().rsd_set_prompts(ctx.handle, _dev_ptr(tokens_dev), _np_ptr(pl)))


def rsd_set_uniforms(ctx: Context, u_draft=None, u_target=None, u_gate=None) -> None:
    for u, cols in ((u_draft, ctx.max_ctx), (u_target, ctx.max_ctx), (u_gate, ctx.max_steps)):
        assert u is None or tuple(u.shape) == (ctx.batch, cols) and u.is_contiguous()
    ctx.keep["uniforms"] = (u_draft, u_target, u_gate)
    ctx.check(load_library().rsd_set_uniforms(ctx.handle, _dev_ptr(u_draft), _dev_ptr(u_target), _dev_ptr(u_gate)))


def rsd_set_criterion(ctx: Context, delta: float, omega_kind: int = 0, omega_a: float = 0.0) -> None:
    ctx.check(load_library().rsd_set_criterion(ctx.handle, C.c_float(delta), C.c_int32(omega_kind), C.c_float(omega_a)))


def rsd_set_teacher(ctx: Context, forced_draft=None, forced_target=None, forced_accept=None) -> None:
    ctx.keep["teacher"] = (forced_draft, forced_target, forced_accept)
    ctx.check(load_library().rsd_set_teacher(ctx.handle, _dev_ptr(forced_draft), _dev_ptr(forced_target),
                                             _dev_ptr(forced_accept)))


def rsd_step(ctx: Context) -> dict:
    B, cap = ctx.batch, ctx.step_cap
    o = dict(draft_len=np.zeros(B, np.int32), draft_tokens=np.full((B, cap), -1, np.int32),
             reward=np.zeros(B, np.float32), accepted=np.zeros(B, np.int32), own_accept=np.zeros(B, np.int32),
             final_len=np.zeros(B, np.int32), final_tokens=np.full((B, cap), -1, np.int32),
             finished=np.zeros(B, np.int32), sd_rounds=np.zeros(B, np.int32), sd_proposed=np.zeros(B, np.int32),
             sd_kept=np.zeros(B, np.int32))
    so = _StepOut(*[_np_ptr(o[n]) for n, _ in _StepOut._fields_])
    ctx.check(load_library().rsd_step(ctx.handle, C.byref(so)))
    return o


def rsd_generate(ctx: Context, max_steps: int = 0, want_tokens: bool = True) -> dict:
    B = ctx.batch
    toks = np.zeros((B, ctx.max_ctx), np.int32) if want_tokens else None
    cl, fin = np.zeros(B, np.int32), np.zeros(B, np.int32)
    g = _GenOut(_np_ptr(toks), _np_ptr(cl), _np_ptr(fin), 0, 0, 0, 0, 0, 0, 0, 0, 0)
    rc = load_library().rsd_generate(ctx.handle, C.c_int32(max_steps), C.byref(g))
    out = dict(tokens=toks, ctx_len=cl, finished=fin, steps_run=g.steps_run, n_committed=g.n_committed,
               n_draft=g.n_draft, n_target=g.n_target, n_accept=g.n_accept, n_reject=g.n_reject, n_sd_rounds=g.n_sd_rounds,
               n_sd_proposed=g.n_sd_proposed, n_sd_kept=g.n_sd_kept, rc=rc)
    ctx.check(rc)
    return out


def rsd_bon_step(ctx: Context) -> dict:
    """One step of process Best-of-N; arrays are per sequence, candidate arrays [sequences, N, ...]."""
    S, N, cap = ctx.n_seq, ctx.bon_n, ctx.step_cap
    o = dict(cand_len=np.zeros((S, N), np.int32), cand_tokens=np.full((S, N, cap), -1, np.int32),
             cand_reward=np.zeros((S, N), np.float32), chosen=np.zeros(S, np.int32), own_choice=np.zeros(S, np.int32),
             finished=np.zeros(S, np.int32), ctx_len=np.zeros(S, np.int32), kv_len=np.zeros((2, S), np.int32),
             n_pages=np.zeros((2, S), np.int32))
    bo = _BonOut(*[_np_ptr(o[n]) for n, _ in _BonOut._fields_])
    ctx.check(load_library().rsd_bon_step(ctx.handle, C.byref(bo)))
    return o


def rsd_bon_generate(ctx: Context, max_steps: int = 0, want_tokens: bool = True) -> dict:
    S = ctx.n_seq
    toks = np.zeros((S, ctx.max_ctx), np.int32) if want_tokens else None
    cl, fin = np.zeros(S, np.int32), np.zeros(S, np.int32)
    g = _GenOut(_np_ptr(toks), _np_ptr(cl), _np_ptr(fin), 0, 0, 0, 0, 0, 0, 0, 0, 0)
    rc = load_library().rsd_bon_generate(ctx.handle, C.c_int32(max_steps), C.byref(g))
    ctx.check(rc)
    return dict(tokens=toks, ctx_len=cl, finished=fin, steps_run=g.steps_run, n_committed=g.n_committed, n_draft=g.n_draft)


def rsd_bon_stats(ctx: Context) -> dict:
    a, b, d = C.c_int64(), C.c_int64(), C.c_int64()
    ctx.check(load_library().rsd_bon_stats(ctx.handle, C.byref(a), C.byref(b), C.byref(d)))
    return dict(pages_shared=a.value, pages_copied=b.value, pages_allocated=d.value)


def rsd_export_state(ctx: Context, want_tokens: bool = True) -> dict:
    B = ctx.batch
    cl, kv, npg = np.zeros(B, np.int32), np.zeros((3, B), np.int32), np.zeros((3, B), np.int32)
    toks = np.zeros((B, ctx.max_ctx), np.int32) if want_tokens else None
    ctx.check(load_library().rsd_export_state(ctx.handle, _np_ptr(cl), _np_ptr(kv), _np_ptr(npg), _np_ptr(toks)))
    return dict(ctx_len=cl, kv_len=kv, n_pages=npg, tokens=toks)


def rsd_export_pages(ctx: Context, model: int) -> dict:
    mp, pp, fp = C.c_int32(), C.c_int32(), C.c_int32()
    lib = load_library()
    ctx.check(lib.rsd_export_pages(ctx.handle, C.c_int32(model), None, C.byref(mp), C.byref(pp), C.byref(fp)))
    bt = np.zeros((ctx.batch, mp.value), np.int32)
    ctx.check(lib.rsd_export_pages(ctx.handle, C.c_int32(model), _np_ptr(bt), None, None, None))
    return dict(block_table=bt, max_pages=mp.value, pool_pages=pp.value, free_pages=fp.value)


def rsd_export_sampled(ctx: Context):
    a = np.zeros((ctx.batch, ctx.max_steps, ctx.step_cap), np.int32)
    b = np.zeros((ctx.batch, ctx.max_steps, ctx.step_cap), np.int32)
    ctx.check(load_library().rsd_export_sampled(ctx.handle, _np_ptr(a), _np_ptr(b)))
    return a, b


def rsd_set_teacher_sd(ctx: Context, forced_proposal=None) -> None:
    ctx.keep["teacher_sd"] = forced_proposal
    ctx.check(load_library().rsd_set_teacher_sd(ctx.handle, _dev_ptr(forced_proposal)))


def rsd_export_proposed(ctx: Context, want_flags: bool = False):
    a = np.zeros((ctx.batch, ctx.max_steps, ctx.step_cap * ctx.sd_k), np.int32)
    f = np.zeros_like(a) if want_flags else None
    ctx.check(load_library().rsd_export_proposed(ctx.handle, _np_ptr(a), _np_ptr(f)))
    return (a, f) if want_flags else a


def rsd_set_uniforms_sd(ctx: Context, u_proposal=None, u_accept=None) -> None:
    for u in (u_proposal, u_accept):
        assert u is None or tuple(u.shape) == (ctx.batch, ctx.max_ctx)
    ctx.keep["uniforms_sd"] = (u_proposal, u_accept)
    ctx.check(load_library().rsd_set_uniforms_sd(ctx.handle, _dev_ptr(u_proposal), _dev_ptr(u_accept)))


def rsd_sd_verify(ctx: Context, p_logits, q_logits, proposals, n_proposals: np.ndarray, u_accept, u_new):
    """The sampled verification rule on given logits: returns (emitted [n, sd_k+1], kept [n]) as numpy."""
    import torch
    n, k = int(p_logits.shape[0]), ctx.sd_k
    assert tuple(p_logits.shape) == (n, k + 1, ctx.vocab) and tuple(q_logits.shape) == (n, k, ctx.vocab)
    assert tuple(proposals.shape) == (n, k) and tuple(u_accept.shape) == (n, k + 1) and tuple(u_new.shape) == (n, k + 1)
    assert p_logits.dtype == torch.float32 and q_logits.dtype == torch.float32 and proposals.dtype == torch.int32
    cnt = np.ascontiguousarray(n_proposals, dtype=np.int32)
    em = torch.full((n, k + 1), -1, dtype=torch.int32, device=p_logits.device)
    kept = torch.zeros(n, dtype=torch.int32, device=p_logits.device)
    ctx.check(load_library().rsd_sd_verify(ctx.handle, _dev_ptr(p_logits), _dev_ptr(q_logits), _dev_ptr(proposals), _np_ptr(cnt),
                                           _dev_ptr(u_accept), _dev_ptr(u_new), C.c_int32(n), _dev_ptr(em), _dev_ptr(kept)))
    return em.cpu().numpy(), kept.cpu().numpy()


def rsd_forward(ctx: Context, model: int, tokens: np.ndarray, lens: np.ndarray, chunk: int):
    """Teacher-forced logits ``[B, T, vocab]`` (LM models) or rewards ``[B, T]``
    as a device tensor; positions beyond ``lens`` hold NaN."""
    import torch

    tokens = np.ascontiguousarray(tokens, dtype=np.int32)
    lens = np.ascontiguousarray(lens, dtype=np.int32)
    B, T = tokens.shape
    assert B == ctx.batch
    shape = (B, T, ctx.vocab) if model != RSD_PRM else (B, T)
    out = torch.full(shape, float("nan"), dtype=torch.float32, device="cuda")
    torch.cuda.current_stream().synchronize()
    ctx.check(load_library().rsd_forward(ctx.handle, C.c_int32(model), _np_ptr(tokens), _np_ptr(lens), C.c_int32(T),
                                         C.c_int32(chunk), _dev_ptr(out)))
    return out


def rsd_sample(ctx: Context, logits, u, temperature: float, top_p: float):
    import torch

    n, V = logits.shape
    out = torch.empty(n, dtype=torch.int32, device=logits.device)
    torch.cuda.current_stream().synchronize()
    ctx.check(load_library().rsd_sample(ctx.handle, _dev_ptr(logits), _dev_ptr(u), C.c_int32(n), C.c_int32(V),
                                        C.c_float(temperature), C.c_float(top_p), _dev_ptr(out)))
    return out


def rsd_sample_static(logits, u, temperature: float, top_p: float, out=None, stream=None):
    """The sampler through the entry point that allocates nothing: ``out`` (device int32 [n]) is the caller's;
    nothing is synchronised (the result is valid once ``stream`` has reached the kernels)."""
    import torch

    n, V = logits.shape
    if out is None:
        out = torch.empty(n, dtype=torch.int32, device=logits.device)
    st = stream if stream is not None else torch.cuda.current_stream()
    rc = load_library().rsd_sample_static(_dev_ptr(logits), _dev_ptr(u), C.c_int32(n), C.c_int32(V), C.c_float(temperature),
                                          C.c_float(top_p), _dev_ptr(out), C.c_void_p(st.cuda_stream))
    if rc != RSD_OK:
        raise RsdError(rc, "rsd_sample_static failed (bad argument, more rows than the static workspace holds, or a HIP error)")
    return out


def rsd_stage_ms(ctx: Context, reset: bool = False) -> np.ndarray:
    ms = (C.c_double * 4)()
    ctx.check(load_library().rsd_stage_ms(ctx.handle, ms, C.c_int32(int(reset))))
    return np.array(list(ms))


def rsd_decode_stats(ctx: Context) -> dict:
    a, b, g = C.c_int64(), C.c_int64(), C.c_int64()
    ctx.check(load_library().rsd_decode_stats(ctx.handle, C.byref(a), C.byref(b), C.byref(g)))
    return dict(eager_iters=a.value, graph_replays=b.value, graphs_recorded=g.value)


def rsd_probe_start(ctx: Context, slot: int, model: int, phase: int, op: int, max_samples: int = 4096, stride: int = 1) -> None:
    ctx.check(load_library().rsd_probe_start(ctx.handle, C.c_int32(slot), C.c_int32(model), C.c_int32(phase), C.c_int32(op),
                                             C.c_int32(max_samples), C.c_int32(stride)))


def rsd_probe_read(ctx: Context, slot: int) -> dict:
    n, ms, by, fl = C.c_int64(), C.c_double(), C.c_int64(), C.c_int64()
    ctx.check(load_library().rsd_probe_read(ctx.handle, C.c_int32(slot), C.byref(n), C.byref(ms), C.byref(by), C.byref(fl)))
    return dict(n=n.value, total_ms=ms.value, total_bytes=by.value, total_flops=fl.value)


def rsd_probe_clock(ctx: Context, slot: int) -> dict:
    n, sh, ref = C.c_int64(), C.c_int64(), C.c_int64()
    ctx.check(load_library().rsd_probe_clock(ctx.handle, C.c_int32(slot), C.byref(n), C.byref(sh), C.byref(ref)))
    return dict(launches=n.value, shader_ticks=sh.value, ref_ticks=ref.value)


def rsd_iter_rows(ctx: Context, model: int) -> int:
    n = C.c_int64()
    ctx.check(load_library().rsd_iter_rows(ctx.handle, C.c_int32(model), C.byref(n)))
    return n.value


def rsd_iter_stats(ctx: Context, model: int, reset: bool = False) -> dict:
    """The counters of rsd_iter_stats, with rsd_iter_rows' count (read first: a reset clears both)."""
    rows = rsd_iter_rows(ctx, model)
    it, ms, si, kv = C.c_int64(), C.c_double(), C.c_int64(), C.c_int64()
    ctx.check(load_library().rsd_iter_stats(ctx.handle, C.c_int32(model), C.byref(it), C.byref(ms), C.byref(si), C.byref(kv),
                                            C.c_int32(int(reset))))
    return dict(iterations=it.value, gpu_ms=ms.value, seq_iterations=si.value, kv_tokens_read=kv.value, row_iterations=rows)


def rsd_check_rows(ctx: Context, model: int, seq: np.ndarray, pos: np.ndarray) -> None:
    """Raises RsdError (RSD_ESTATE) when a pass over rows (seq[i], pos[i]) would leave the pages of ``model``."""
    s = np.ascontiguousarray(seq, dtype=np.int32)
    p = np.ascontiguousarray(pos, dtype=np.int32)
    assert s.shape == p.shape and s.ndim == 1
    ctx.check(load_library().rsd_check_rows(ctx.handle, C.c_int32(model), _np_ptr(s), _np_ptr(p), C.c_int32(s.size)))


def rsd_debug_build() -> bool:
    return bool(load_library().rsd_debug_build())


def rsd_probe_attention(ctx: Context, model: int, ctx_len: np.ndarray, reps: int) -> float:
    """Milliseconds for ``reps`` launches of the decode attention of ``model`` over contexts ``ctx_len``."""
    cl = np.ascontiguousarray(ctx_len, dtype=np.int32)
    assert cl.shape == (ctx.batch,)
    ms = C.c_double()
    ctx.check(load_library().rsd_probe_attention(ctx.handle, C.c_int32(model), _np_ptr(cl), C.c_int32(reps), C.byref(ms)))
    return ms.value


# the operators of include/rsd_ops.h (they use this module's library and errors)
from .ops import *  # noqa: E402,F401,F403
from .ops import __all__ as _ops_all  # noqa: E402

__all__ += _ops_all
