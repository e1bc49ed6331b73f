"""ctypes binding of include/disco.h: the same entry points under the same names, plus small
holders that keep the PyTorch-allocated device buffers of a model, a KV cache and a workspace alive.
No arithmetic of the method happens here."""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdisco.so")

MAX_BLOCK = 16
N_FEAT = 12
FAMILY = {"A": 0, "B": 1}
OK, EINVAL, ECAP, ESTATE, EHIP = 0, -1, -2, -3, -4


class DiscoError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"disco error {code}: {msg}")
        self.code = code


class ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("family", "n_layers", "d_model", "n_heads", "d_head",
                                         "n_kv_heads", "d_ff", "vocab", "max_pos")] + \
               [("norm_eps", C.c_float), ("rope_base", C.c_float)]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("norm1_g", "norm1_b", "wqkv", "wo", "norm2_g", "norm2_b",
                                          "w_in", "w_out")]


class ModelWeights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("tok_emb_stride", C.c_int64), ("pos_emb", C.c_void_p),
                ("layers", C.POINTER(LayerWeights)), ("normf_g", C.c_void_p), ("normf_b", C.c_void_p),
                ("wlm", C.c_void_p)]


class Clf(C.Structure):
    _fields_ = [("dev_params", C.c_void_p), ("hidden", C.c_int32)]


class ClfOut(C.Structure):
    _fields_ = [("token", C.c_int32), ("feats", C.c_float * N_FEAT), ("score", C.c_float),
                ("halt", C.c_uint32), ("executed", C.c_uint32)]


class AcceptOut(C.Structure):
    _fields_ = [("n", C.c_int32), ("n_emit", C.c_int32), ("emit", C.c_int32 * MAX_BLOCK)]


class LoopOpts(C.Structure):
    _fields_ = [("dev_force_tokens", C.c_void_p), ("dev_ref_tokens", C.c_void_p), ("temperature", C.c_float),
                ("dev_u_draft", C.c_void_p), ("dev_draft_probs", C.c_void_p), ("ppl_threshold", C.c_float),
                ("block_offset", C.c_int32), ("open_end", C.c_int32)]


class LoopOut(C.Structure):
    _fields_ = [("sl", C.c_int32), ("block", C.c_int32 * MAX_BLOCK), ("halted", C.c_int32)]


class IterBuffers(C.Structure):
    _fields_ = [("dev_tokens_in", C.c_void_p), ("dev_logits_draft", C.c_void_p), ("dev_steps", C.c_void_p),
                ("dev_loop_out", C.c_void_p), ("host_loop_out", C.c_void_p), ("dev_argmax", C.c_void_p),
                ("dev_accept_out", C.c_void_p), ("host_accept_out", C.c_void_p)]


class IterResult(C.Structure):
    _fields_ = [("sl", C.c_int32), ("n", C.c_int32), ("draft_forwards", C.c_int32),
                ("draft_steps_enqueued", C.c_int32), ("block", C.c_int32 * MAX_BLOCK), ("emit", C.c_int32 * MAX_BLOCK)]


class SharedKVDesc(C.Structure):
    _fields_ = [("dev_prefix", C.c_void_p), ("dev_prefix_table", C.c_void_p), ("n_prefix_pages", C.c_int32), ("prefix_len", C.c_int32),
                ("dev_pages", C.c_void_p), ("dev_tables", C.c_void_p), ("dev_lens", C.c_void_p), ("n_pages", C.c_int32),
                ("table_ld", C.c_int32), ("n_seqs", C.c_int32), ("page_tokens", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32)]


_SIGNATURES = {
    "disco_last_error": (C.c_char_p, []),
    "disco_pack_weight": (C.c_int, [C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p]),
    "disco_pack_gate_up": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p]),
    "disco_model_create": (C.c_int, [C.POINTER(ModelDesc), C.POINTER(ModelWeights), C.POINTER(C.c_void_p)]),
    "disco_model_destroy": (None, [C.c_void_p]),
    "disco_kv_bytes": (C.c_size_t, [C.c_void_p, C.c_int, C.c_int]),
    "disco_kv_create": (C.c_int, [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int, C.c_int,
                                  C.POINTER(C.c_int32), C.POINTER(C.c_void_p)]),
    "disco_kv_destroy": (None, [C.c_void_p]),
    "disco_kv_len": (C.c_int, [C.c_void_p]),
    "disco_kv_pages_in_use": (C.c_int, [C.c_void_p]),
    "disco_kv_fill": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]),
    "disco_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int, C.c_int]),
    "disco_workspace_init": (C.c_int, [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int, C.c_int, C.c_void_p]),
    "disco_prefill_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int, C.c_int]),
    "disco_prefill": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_size_t,
                                C.c_void_p]),
    "disco_prefill_ex": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_uint, C.c_void_p,
                                   C.c_size_t, C.c_void_p]),
    "disco_draft_step": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                                   C.c_size_t, C.c_void_p, C.c_void_p]),
    "disco_classify": (C.c_int, [C.POINTER(Clf), C.c_void_p, C.c_int, C.c_float, C.c_float, C.c_int,
                                 C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_void_p, C.c_void_p]),
    "disco_classify_scratch_init": (C.c_int, [C.c_void_p, C.c_void_p]),
    "disco_classify_static": (C.c_int, [C.POINTER(Clf), C.c_void_p, C.c_int, C.c_float, C.c_float, C.c_int,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_void_p]),
    "disco_verify": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                               C.c_void_p, C.c_size_t, C.c_void_p]),
    "disco_accept": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                               C.c_void_p]),
    "disco_kv_rollback": (C.c_int, [C.c_void_p, C.c_int]),
    "disco_draft_loop": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(Clf), C.c_void_p, C.c_int, C.c_int,
                                   C.c_int, C.c_float, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "disco_sample": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int64, C.c_float, C.c_void_p, C.c_void_p,
                               C.c_void_p, C.c_void_p]),
    "disco_accept_sample": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                      C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "disco_draft_loop_sampled": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(Clf), C.c_void_p, C.c_int, C.c_int,
                                           C.c_int, C.c_float, C.c_float, C.c_float, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_size_t, C.c_void_p]),
    "disco_draft_loop_ex": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(Clf), C.c_void_p, C.c_int, C.c_int,
                                      C.c_int, C.c_float, C.c_float, C.POINTER(LoopOpts), C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "disco_iterate": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p,
                                C.c_size_t, C.POINTER(Clf), C.POINTER(C.c_int32), C.c_int, C.c_int, C.c_int, C.c_int,
                                C.c_float, C.c_float, C.POINTER(LoopOpts), C.POINTER(IterBuffers),
                                C.POINTER(IterResult), C.c_void_p]),
    "disco_clf_train": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_float, C.c_void_p,
                                  C.c_void_p, C.c_void_p]),
    "disco_clf_eval": (C.c_int, [C.POINTER(Clf), C.c_void_p, C.c_void_p, C.c_int, C.c_float, C.c_void_p,
                                 C.c_void_p, C.c_void_p]),
    "disco_set_launch_mode": (C.c_int, [C.c_int]),
    "disco_rope_table": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_float, C.c_void_p]),
    "disco_append": (C.c_int, [C.POINTER(SharedKVDesc), C.c_void_p, C.c_int, C.c_int64, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                               C.c_int, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_int64, C.c_void_p]),
    "disco_attn_shared_bytes": (C.c_size_t, [C.POINTER(SharedKVDesc), C.c_int, C.c_int, C.c_int]),
    "disco_attn_shared": (C.c_int, [C.POINTER(SharedKVDesc), C.c_void_p, C.c_int, C.c_int64, C.c_int, C.c_int, C.c_float, C.c_void_p, C.c_int64,
                                    C.c_void_p, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "disco_beam_select_bytes": (C.c_size_t, [C.c_int, C.c_int, C.c_int, C.c_int]),
    "disco_beam_select": (C.c_int, [C.c_void_p, C.c_int, C.c_int64, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_int,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "disco_step_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_void_p, C.POINTER(SharedKVDesc)]),
    "disco_step": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(SharedKVDesc), C.c_int64, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                             C.c_void_p]),
    "disco_beam_reorder": (C.c_int, [C.c_void_p, C.c_int, C.c_int64, C.c_int, C.c_int64, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int,
                                     C.c_int, C.c_int, C.c_int, C.c_void_p]),
    "disco_clf_examples": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "disco_heuristic_next": (C.c_int, [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int]),
    "disco_probe_enable": (C.c_int, [C.c_int]),
    "disco_probe_read_ms": (C.c_float, []),
    "disco_set_wait_limit": (C.c_int, [C.c_int]),
    "disco_qkv_attn_plan": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int)]),
    "disco_layers_plan": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int)]),
    "disco_forward_route": (C.c_int, []),
    "disco_prefill_plan": (C.c_int, [C.c_void_p, C.c_int, C.c_uint, C.c_int, C.POINTER(C.c_int)]),
}
EXPORTS = sorted(_SIGNATURES)

_lib = None


def lib() -> C.CDLL:
    """The loaded library.  Fails loudly when it has not been built: there is no fallback path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2405_04304_amd.build` "
                               "(there is no CPU or PyTorch fallback for the DISCO kernels)")
        _lib = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(_lib, name)
            fn.restype, fn.argtypes = res, args
    return _lib


def last_error() -> str:
    return lib().disco_last_error().decode()


def _check(rc: int) -> None:
    if rc != 0:
        raise DiscoError(rc, last_error())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# ---- the C entry points, same names, tensors or raw addresses accepted -----------------------

def disco_pack_weight(src, n, k, dst, stream=None):
    _check(lib().disco_pack_weight(_ptr(src), n, k, _ptr(dst), _stream() if stream is None else stream))


def disco_pack_gate_up(gate, up, d_ff, k, dst, stream=None):
    _check(lib().disco_pack_gate_up(_ptr(gate), _ptr(up), d_ff, k, _ptr(dst),
                                    _stream() if stream is None else stream))


def disco_draft_step(model, kv, tokens_in, n_in, logits, ws, gate=None, stream=None):
    _check(lib().disco_draft_step(model.handle, kv.handle, _ptr(tokens_in), n_in, _ptr(logits),
                                  _ptr(ws.buf), ws.nbytes, _ptr(gate),
                                  _stream() if stream is None else stream))


def disco_classify(clf, logits, vocab, pos_feature, tau, force_halt, out, token_next=None,
                   block_slot=None, gate=None, sl_count=None, force_token=None, scratch=None, stream=None):
    _check(lib().disco_classify(C.byref(clf.c) if clf is not None else None, _ptr(logits), vocab,
                                pos_feature, tau, int(force_halt), _ptr(out), _ptr(token_next),
                                _ptr(block_slot), _ptr(gate), _ptr(sl_count), _ptr(force_token), _ptr(scratch),
                                _stream() if stream is None else stream))


def disco_classify_static(clf, logits, vocab, pos_feature, tau, force_halt, out, token_next=None,
                          block_slot=None, gate=None, sl_count=None, force_token=None, stream=None):
    _check(lib().disco_classify_static(C.byref(clf.c) if clf is not None else None, _ptr(logits), vocab,
                                       pos_feature, tau, int(force_halt), _ptr(out), _ptr(token_next),
                                       _ptr(block_slot), _ptr(gate), _ptr(sl_count), _ptr(force_token),
                                       _stream() if stream is None else stream))


CLASSIFY_SCRATCH_BYTES = 4352


def classify_scratch(device="cuda") -> torch.Tensor:
    """Device scratch for the many-workgroup form of disco_classify, ticket word zeroed."""
    t = torch.empty(CLASSIFY_SCRATCH_BYTES, dtype=torch.uint8, device=device)
    _check(lib().disco_classify_scratch_init(t.data_ptr(), _stream()))
    return t


def disco_verify(model, kv, block, n_block, argmax, logits, ws, stream=None):
    _check(lib().disco_verify(model.handle, kv.handle, _ptr(block), n_block, _ptr(argmax), _ptr(logits),
                              _ptr(ws.buf), ws.nbytes, _stream() if stream is None else stream))


PREFILL_BF16_ACTIVATIONS = 1


def disco_prefill(model, kv, tokens, n_tokens, logits_last, ws, stream=None, flags=0):
    if flags:
        _check(lib().disco_prefill_ex(model.handle, kv.handle, _ptr(tokens), n_tokens, _ptr(logits_last), flags,
                                      _ptr(ws.buf), ws.nbytes, _stream() if stream is None else stream))
        return
    _check(lib().disco_prefill(model.handle, kv.handle, _ptr(tokens), n_tokens, _ptr(logits_last), _ptr(ws.buf),
                               ws.nbytes, _stream() if stream is None else stream))


def disco_accept(block, argmax, n_block, out, host_out=None, dev_n_block=None, stream=None):
    _check(lib().disco_accept(_ptr(block), _ptr(argmax), n_block, _ptr(dev_n_block), _ptr(out),
                              _ptr(host_out), _stream() if stream is None else stream))


def disco_kv_rollback(kv, new_len):
    _check(lib().disco_kv_rollback(kv.handle, new_len))


def disco_draft_loop(model, kv, clf, tokens_in, n_in, cap, static_sl, pos_feature0, tau, force_tokens,
                     logits, steps, out, host_out, ws, stream=None):
    _check(lib().disco_draft_loop(model.handle, kv.handle, C.byref(clf.c) if clf is not None else None,
                                  _ptr(tokens_in), n_in, cap, static_sl, pos_feature0, tau,
                                  _ptr(force_tokens), _ptr(logits), _ptr(steps), _ptr(out),
                                  _ptr(host_out), _ptr(ws.buf), ws.nbytes,
                                  _stream() if stream is None else stream))


def disco_draft_loop_ex(model, kv, clf, tokens_in, n_in, cap, static_sl, pos_feature0, tau, logits, steps, out,
                        host_out, ws, force_tokens=None, ref_tokens=None, temperature=0.0, u_draft=None,
                        draft_probs=None, ppl_threshold=0.0, block_offset=0, open_end=0, stream=None):
    opts = LoopOpts(_ptr(force_tokens), _ptr(ref_tokens), temperature, _ptr(u_draft), _ptr(draft_probs),
                    ppl_threshold, block_offset, open_end)
    _check(lib().disco_draft_loop_ex(model.handle, kv.handle, C.byref(clf.c) if clf is not None else None,
                                     _ptr(tokens_in), n_in, cap, static_sl, pos_feature0, tau, C.byref(opts),
                                     _ptr(logits), _ptr(steps), _ptr(out), _ptr(host_out), _ptr(ws.buf), ws.nbytes,
                                     _stream() if stream is None else stream))


def iter_buffers(tokens_in, logits_draft, steps, loop_out, host_loop_out, argmax, accept_out, host_accept_out):
    return IterBuffers(_ptr(tokens_in), _ptr(logits_draft), _ptr(steps), _ptr(loop_out), _ptr(host_loop_out),
                       _ptr(argmax), _ptr(accept_out), _ptr(host_accept_out))


def disco_iterate(target, kv_t, ws_t, draft, kv_d, ws_d, clf, pending, cap, static_sl, chunk, pos_feature0, tau,
                  buffers, result, force_tokens=None, ref_tokens=None, ppl_threshold=0.0, stream=None):
    """One speculative iteration in the library; `result` (IterResult) is filled on return."""
    opts = LoopOpts(_ptr(force_tokens), _ptr(ref_tokens), 0.0, None, None, ppl_threshold, 0, 0)
    pend = (C.c_int32 * len(pending))(*pending)
    _check(lib().disco_iterate(target.handle, kv_t.handle, _ptr(ws_t.buf), ws_t.nbytes,
                               draft.handle if draft is not None else None, kv_d.handle if kv_d is not None else None,
                               _ptr(ws_d.buf) if ws_d is not None else None, ws_d.nbytes if ws_d is not None else 0,
                               C.byref(clf.c) if clf is not None else None, pend, len(pending), cap, static_sl, chunk,
                               pos_feature0, tau, C.byref(opts), C.byref(buffers), C.byref(result),
                               _stream() if stream is None else stream))


def disco_sample(logits, n_rows, vocab, ld_logits, temperature, u, probs, tokens, stream=None):
    _check(lib().disco_sample(_ptr(logits), n_rows, vocab, ld_logits, temperature, _ptr(u), _ptr(probs),
                              _ptr(tokens), _stream() if stream is None else stream))


def disco_accept_sample(block, n_block, draft_probs, target_logits, vocab, temperature, u_accept, u_resample,
                        out, host_out=None, dev_n_block=None, stream=None):
    _check(lib().disco_accept_sample(_ptr(block), n_block, _ptr(dev_n_block), _ptr(draft_probs),
                                     _ptr(target_logits), vocab, temperature, _ptr(u_accept), _ptr(u_resample),
                                     _ptr(out), _ptr(host_out), _stream() if stream is None else stream))


def disco_draft_loop_sampled(model, kv, clf, tokens_in, n_in, cap, static_sl, pos_feature0, tau, temperature,
                             u_draft, draft_probs, logits, steps, out, host_out, ws, stream=None):
    _check(lib().disco_draft_loop_sampled(model.handle, kv.handle, C.byref(clf.c) if clf is not None else None,
                                          _ptr(tokens_in), n_in, cap, static_sl, pos_feature0, tau, temperature,
                                          _ptr(u_draft), _ptr(draft_probs), _ptr(logits), _ptr(steps), _ptr(out),
                                          _ptr(host_out), _ptr(ws.buf), ws.nbytes,
                                          _stream() if stream is None else stream))


# ---- several sequences that continue one prompt ------------------------------------------------

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _refuse(what: str):
    raise DiscoError(EINVAL, what)


def _bad_tensor(t, what, dtype, numel):
    """Says why _tensor refused (built only then: a decoding step makes these checks dozens of times)."""
    if t is None:
        _refuse(f"{what} is missing")
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        _refuse(f"{what} is not on the current device")
    if t.dtype is not dtype:
        _refuse(f"{what} has type {t.dtype}, not {dtype}")
    if not t.is_contiguous():
        _refuse(f"{what} is not contiguous")
    _refuse(f"{what} has {t.numel()} elements, {numel} needed")


def _device() -> int:
    """The current device, -1 where there is none (what torch.cuda.current_device asks, without its checks)."""
    try:
        return torch._C._cuda_getDevice()
    except RuntimeError:
        return -1


def _tensor(t, what: str, dev: int, dtype, numel: int = 0) -> int:
    """Address of a tensor, after the checks that the library cannot make: device, type, contiguous, size."""
    if t is None or not t.is_cuda or t.get_device() != dev or t.dtype is not dtype or not t.is_contiguous() or t.numel() < numel:
        _bad_tensor(t, what, dtype, numel)
    return t.data_ptr()


def _rows(t, what: str, dev: int, n: int, width: int):
    """(address, element type code, row stride) of a matrix of n rows whose columns are contiguous."""
    if not t.is_cuda or t.get_device() != dev:
        _refuse(f"{what} is not on the current device")
    code = _DTYPES.get(t.dtype)
    if code is None:
        _refuse(f"{what} has type {t.dtype}: float32 or bfloat16")
    shape = t.shape
    if len(shape) != 2 or shape[0] < n or shape[1] < width:
        _refuse(f"{what} has shape {tuple(shape)}, ({n}, {width}) needed")
    ld, one = t.stride()
    if one != 1 and shape[1] != 1:
        _refuse(f"{what}: the elements of a row are not contiguous")
    return t.data_ptr(), code, ld if n > 1 else max(ld, shape[1])


def _raw_stream(dev: int, stream) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream


class SharedKV:
    """One layer of the paged cache of several sequences behind one prompt (disco_shared_kv); keeps its tensors alive.

    pages, prefix_pages: bf16 [pages, 2, n_kv_heads, page_tokens * d_head]; tables: int32 [n_seqs, pages a table holds]; lens: int32
    [n_seqs] (None if every append names its rows' positions); prefix_table: int32 or None (page i of the prompt is page i)."""

    def __init__(self, pages, tables, lens, page_tokens: int, n_kv_heads: int, d_head: int, prefix_pages=None, prefix_len: int = 0,
                 prefix_table=None):
        page_shape, dev = (2, n_kv_heads, page_tokens * d_head), _device()
        _tensor(pages, "pages", dev, torch.bfloat16)
        if pages.dim() != 4 or tuple(pages.shape[1:]) != page_shape:
            _refuse(f"pages have shape {tuple(pages.shape)}, (pages, {page_shape}) needed")
        _tensor(tables, "tables", dev, torch.int32)
        if tables.dim() != 2:
            _refuse("tables: [sequences, pages]")
        if lens is not None:
            _tensor(lens, "lens", dev, torch.int32, tables.shape[0])
        n_prefix = 0
        if prefix_pages is not None:
            _tensor(prefix_pages, "prefix_pages", dev, torch.bfloat16)
            if prefix_pages.dim() != 4 or tuple(prefix_pages.shape[1:]) != page_shape:
                _refuse("prefix_pages have another page shape")
            n_prefix = prefix_pages.shape[0]
            if prefix_table is not None:
                _tensor(prefix_table, "prefix_table", dev, torch.int32, -(-prefix_len // page_tokens))
        self._keep = (pages, tables, lens, prefix_pages, prefix_table)
        self.lens = lens
        self.n_seqs, self.n_kv_heads, self.d_head = tables.shape[0], n_kv_heads, d_head
        self.c = SharedKVDesc(_ptr(prefix_pages), _ptr(prefix_table), n_prefix, prefix_len, _ptr(pages), _ptr(tables), _ptr(lens),
                              pages.shape[0], tables.shape[1], tables.shape[0], page_tokens, n_kv_heads, d_head)
        self.ref = C.byref(self.c)


def disco_rope_table(n_pos: int, d_head: int, base: float = 10000.0, device="cuda", stream=None) -> torch.Tensor:
    """fp32 [n_pos, d_head / 2, 2]: (cos, sin) of every position and channel pair."""
    t = torch.empty(max(n_pos, 0), max(d_head // 2, 0), 2, dtype=torch.float32, device=device)
    _tensor(t, "device", _device(), torch.float32)
    _check(lib().disco_rope_table(_ptr(t), n_pos, d_head, base, _stream() if stream is None else stream))
    return t


def disco_append(kv: SharedKV, qkv, n_heads: int, q, seq=None, pos=None, rope=None, q_gain=None, k_gain=None, eps: float = 1e-6,
                 stream=None):
    """Keys and values of the rows of qkv into the cache, queries (normalised, rotated) to q."""
    dev, n, d = _device(), qkv.shape[0], kv.d_head
    p_qkv, code, ld = _rows(qkv, "qkv", dev, n, (n_heads + 2 * kv.n_kv_heads) * d)
    p_q, code_q, ld_q = _rows(q, "q", dev, n, n_heads * d)
    if code != code_q:
        _refuse("q has another type than qkv")
    if rope is not None and (rope.dim() != 3 or rope.shape[1] * 2 != d or rope.shape[2] != 2):
        _refuse(f"rope: [positions, {d // 2}, 2]")
    _check(lib().disco_append(kv.ref, p_qkv, code, ld, n, n_heads, None if seq is None else _tensor(seq, "seq", dev, torch.int32, n),
                              None if pos is None else _tensor(pos, "pos", dev, torch.int32, n),
                              None if rope is None else _tensor(rope, "rope", dev, torch.float32), 0 if rope is None else rope.shape[0],
                              None if q_gain is None else _tensor(q_gain, "q_gain", dev, torch.float32, d),
                              None if k_gain is None else _tensor(k_gain, "k_gain", dev, torch.float32, d), eps, p_q, ld_q,
                              _raw_stream(dev, stream)))


def disco_attn_shared_bytes(kv: SharedKV, n_tok: int, n_heads: int, max_len: int = 0) -> int:
    n = lib().disco_attn_shared_bytes(kv.ref, n_tok, n_heads, max_len)
    if n == 0:
        raise DiscoError(EINVAL, last_error())
    return n


def disco_attn_shared(kv: SharedKV, q, n_tok: int, n_heads: int, out, ws, lse=None, scale: Optional[float] = None, max_len: int = 0,
                      stream=None):
    """Attention of n_tok tokens of every sequence; ws: uint8, disco_attn_shared_bytes of the same arguments.  scale: d_head ** -0.5."""
    dev, n = _device(), kv.n_seqs * n_tok
    p_q, code, ld = _rows(q, "q", dev, n, n_heads * kv.d_head)
    p_out, code_o, ld_o = _rows(out, "out", dev, n, n_heads * kv.d_head)
    if code != code_o:
        _refuse("out has another type than q")
    _check(lib().disco_attn_shared(kv.ref, p_q, code, ld, n_tok, n_heads, kv.d_head ** -0.5 if scale is None else scale, p_out, ld_o,
                                   None if lse is None else _tensor(lse, "lse", dev, torch.float32, n * n_heads), max_len,
                                   _tensor(ws, "ws", dev, torch.uint8), ws.numel(), _raw_stream(dev, stream)))


def disco_beam_select_bytes(n_groups: int, n_beams: int, vocab: int, k: int) -> int:
    n = lib().disco_beam_select_bytes(n_groups, n_beams, vocab, k)
    if n == 0:
        raise DiscoError(EINVAL, last_error())
    return n


def disco_beam_select(logits, scores, n_groups: int, n_beams: int, k: int, tokens, parents, scores_out, ws, done=None, done_out=None,
                      end_token: int = -1, stream=None):
    """The k best (beam, token) of every group; logits: [n_groups * n_beams, vocab]."""
    dev, n, nk = _device(), n_groups * n_beams, n_groups * k
    if logits.dim() != 2:
        _refuse("logits: [rows, vocab]")
    vocab = logits.shape[1]
    p_logits, code, ld = _rows(logits, "logits", dev, n, vocab)
    _check(lib().disco_beam_select(p_logits, code, ld, n_groups, n_beams, vocab, k, _tensor(scores, "scores", dev, torch.float32, n),
                                   None if done is None else _tensor(done, "done", dev, torch.int32, n), end_token,
                                   _tensor(tokens, "tokens", dev, torch.int32, nk), _tensor(parents, "parents", dev, torch.int32, nk),
                                   _tensor(scores_out, "scores_out", dev, torch.float32, nk),
                                   None if done_out is None else _tensor(done_out, "done_out", dev, torch.int32, nk),
                                   _tensor(ws, "ws", dev, torch.uint8), ws.numel(), _raw_stream(dev, stream)))


def disco_beam_reorder(pages, tables, parents, tables_out, n_groups: int, n_beams: int, length: int, page_tokens: int, stream=None):
    """Sequence b goes on from parents[b]; pages: bf16 [layers, pages, 2, n_kv_heads, page_tokens * d_head], layers may be strided."""
    dev = _device()
    if not pages.is_cuda or pages.get_device() != dev:
        _refuse("pages are not on the current device")
    shape = pages.shape
    if len(shape) != 5 or pages.dtype is not torch.bfloat16 or shape[0] == 0 or shape[2] != 2 or page_tokens < 1 or shape[4] % page_tokens:
        _refuse("pages: bfloat16 [layers, pages, 2, K / V heads, page_tokens * d_head]")
    layers, n_pages, _, heads, size = shape
    layer, *page = pages.stride()
    if page != [2 * heads * size, heads * size, size, 1]:
        _refuse("pages: the pages of a layer are not contiguous")
    shape = tables.shape
    if len(shape) != 2 or shape[0] < n_groups * n_beams:
        _refuse("tables: [sequences, pages]")
    rows, cols = shape
    _check(lib().disco_beam_reorder(pages.data_ptr(), layers, layer, n_pages, 2 * heads * size, _tensor(tables, "tables", dev, torch.int32),
                                    _tensor(tables_out, "tables_out", dev, torch.int32, rows * cols), cols,
                                    _tensor(parents, "parents", dev, torch.int32, n_groups * n_beams), n_groups, n_beams, length, page_tokens,
                                    _raw_stream(dev, stream)))


class Sequences:
    """Own pages (of every layer), tables and lengths of n sequences that continue the prompt in a DiscoKV: room for `capacity` positions each.

    pages: bf16 [layers, pages, 2, K / V heads, page_tokens * d_head]; tables: two, for disco_beam_reorder to go from one to the other."""

    def __init__(self, model: "DiscoModel", n: int, capacity: int, page_tokens: int = 16):
        s, dev = model.shape, model.device
        self.n, self.page_tokens, cols = n, page_tokens, -(-capacity // page_tokens)
        self.capacity = cols * page_tokens
        self.pages = torch.empty(s.n_layers, n * cols, 2, s.n_kv_heads, page_tokens * s.d_head, dtype=torch.bfloat16, device=dev)
        self.all_lens = torch.arange(1, self.capacity + 1, dtype=torch.int32, device=dev)[:, None].repeat(1, n).contiguous()
        self.tables = [torch.arange(n * cols, dtype=torch.int32, device=dev).view(n, cols) for _ in range(2)]
        self._kv = [SharedKV(self.pages[0], t, self.all_lens[0], page_tokens, s.n_kv_heads, s.d_head) for t in self.tables]
        self.cur, self.len = 0, 0

    def reset(self):
        """Empty again; every table names pages of its own."""
        t = self.tables[0]
        t.copy_(torch.arange(t.numel(), dtype=torch.int32, device=t.device).view_as(t))
        self.cur = self.len = 0

    @property
    def kv(self) -> SharedKV:
        kv = self._kv[self.cur]
        kv.c.dev_lens = self.all_lens.data_ptr() + 4 * self.n * max(self.len - 1, 0)
        return kv


def disco_step(model, kv_prompt, seqs: Sequences, tokens, logits, ws, stream=None):
    """Feeds one token of every sequence; seqs.len grows by one."""
    dev, vocab = _device(), model.shape.vocab
    seqs.len += 1
    try:
        _check(lib().disco_step(model.handle, kv_prompt.handle, seqs.kv.ref, seqs.pages.stride(0), seqs.len,
                                _tensor(tokens, "tokens", dev, torch.int32, seqs.n), _tensor(logits, "logits", dev, torch.float32, seqs.n * vocab),
                                _ptr(ws.buf), ws.nbytes, _raw_stream(dev, stream)))
    except DiscoError:
        seqs.len -= 1
        raise


def disco_step_reorder(seqs: Sequences, parents, n_groups: int = 1, stream=None):
    """disco_beam_reorder of the sequences, in n_groups groups."""
    if n_groups < 1 or seqs.n % n_groups:
        _refuse(f"{seqs.n} sequences in {n_groups} groups")
    disco_beam_reorder(seqs.pages, seqs.tables[seqs.cur], parents, seqs.tables[1 - seqs.cur], n_groups, seqs.n // n_groups, seqs.len,
                       seqs.page_tokens, stream)
    seqs.cur = 1 - seqs.cur


TRAIN_MAX_N = 2560
PREFILL_MAX = 8192


def disco_clf_train(feats, labels, n, hidden, epochs, lr, params, loss=None, stream=None):
    _check(lib().disco_clf_train(_ptr(feats), _ptr(labels), n, hidden, epochs, lr, _ptr(params), _ptr(loss),
                                 _stream() if stream is None else stream))


def disco_clf_eval(clf, feats, labels, n, tau, scores=None, counts=None, stream=None):
    _check(lib().disco_clf_eval(C.byref(clf.c), _ptr(feats), _ptr(labels), n, tau, _ptr(scores), _ptr(counts),
                                _stream() if stream is None else stream))


def disco_clf_examples(records, n, ref_tokens, feats, labels, tokens=None, stream=None):
    _check(lib().disco_clf_examples(_ptr(records), n, _ptr(ref_tokens), _ptr(feats), _ptr(labels), _ptr(tokens),
                                    _stream() if stream is None else stream))


def disco_heuristic_next(lookahead: int, drafted: int, accepted: int, up: int, down: int, cap: int) -> int:
    r = lib().disco_heuristic_next(lookahead, drafted, accepted, up, down, cap)
    if r < 0:
        raise DiscoError(r, last_error())
    return r


def disco_set_launch_mode(mode: int) -> int:
    prev = lib().disco_set_launch_mode(mode)
    if prev < 0:
        raise DiscoError(prev, last_error())
    return prev


def disco_set_wait_limit(polls: int) -> int:
    return int(lib().disco_set_wait_limit(polls))


def disco_prefill_plan(model_handle, n_tokens: int, flags: int = 0, page_tokens: int = 16) -> dict:
    """The kernels a prompt pass would launch (disco_bench.h): tile codes of its four matrices, attention, LayerNorm, copy rings, 1 / rms."""
    out = (C.c_int * 12)()
    _check(lib().disco_prefill_plan(model_handle, n_tokens, flags, page_tokens, out))
    return {"qkv": out[0], "o": out[1], "mlp_in": out[2], "mlp_out": out[3], "attn_tiles": bool(out[4]), "norm_groups": bool(out[5]),
            "stages": dict(zip(("qkv", "o", "mlp_in", "mlp_out"), out[6:10])), "rms_in_launch": {"qkv": bool(out[10]), "mlp_in": bool(out[11])}}


def disco_qkv_attn_plan(model_handle, n_tokens: int, ctx: int, capacity: int = 0) -> dict:
    """How launch mode 0 runs QKV projection and attention (disco_bench.h): form, deal of the context, workgroups."""
    out = (C.c_int * 5)()
    _check(lib().disco_qkv_attn_plan(model_handle, n_tokens, ctx, capacity, out))
    return {"form": ("separate", "shared", "own")[out[0]], "row_tiles": out[1], "range": out[2], "ranges": out[3], "workgroups": out[4]}


def disco_layers_plan(model_handle, n_tokens: int, ctx: int, page_tokens: int, capacity: int = 0) -> dict:
    """Whether launch mode 0 runs all layers of a forward in one launch (disco_bench.h), and its workgroups."""
    out = (C.c_int * 4)()
    _check(lib().disco_layers_plan(model_handle, n_tokens, ctx, page_tokens, capacity, out))
    return {"one_launch": bool(out[0]), "workgroups": out[1], "groups": out[2], "parts": out[3]}


def disco_forward_route() -> str:
    """How the last forward that this thread sent was launched (disco_bench.h)."""
    return ("phases", "shared", "layers", "cooperative")[lib().disco_forward_route()]


def disco_probe_enable(layer: int) -> None:
    _check(lib().disco_probe_enable(layer))


def disco_probe_read_ms() -> float:
    return float(lib().disco_probe_read_ms())


# ---- holders of device memory ------------------------------------------------------------------

class DiscoModel:
    """Packs a dict of row-major weights (names as in workloads.weight_specs) on the device and owns
    the packed buffers and the library handle."""

    def __init__(self, shape, weights: Dict[str, torch.Tensor], device="cuda", tok_emb=None,
                 tok_emb_stride: Optional[int] = None):
        self.shape = shape
        self.device = torch.device(device)
        self._keep = []
        fam_a = shape.family == "A"

        def dev(t, dtype):
            t = t.to(self.device, dtype=dtype).contiguous()
            self._keep.append(t)
            return t

        def packed(name):
            src = weights[name].to(self.device, dtype=torch.bfloat16).contiguous()
            dst = torch.empty_like(src)
            disco_pack_weight(src, src.shape[0], src.shape[1], dst)
            self._keep.append(dst)
            return dst

        layers = (LayerWeights * shape.n_layers)()
        for l in range(shape.n_layers):
            p = f"l{l}."
            L = layers[l]
            L.norm1_g = dev(weights[p + "norm1_g"], torch.float32).data_ptr()
            L.norm2_g = dev(weights[p + "norm2_g"], torch.float32).data_ptr()
            if fam_a:
                L.norm1_b = dev(weights[p + "norm1_b"], torch.float32).data_ptr()
                L.norm2_b = dev(weights[p + "norm2_b"], torch.float32).data_ptr()
                L.w_in = packed(p + "w1").data_ptr()
                L.w_out = packed(p + "w2").data_ptr()
            else:
                wg = weights[p + "wg"].to(self.device, dtype=torch.bfloat16).contiguous()
                wu = weights[p + "wu"].to(self.device, dtype=torch.bfloat16).contiguous()
                dst = torch.empty((2 * shape.d_ff, shape.d_model), dtype=torch.bfloat16, device=self.device)
                disco_pack_gate_up(wg, wu, shape.d_ff, shape.d_model, dst)
                self._keep.append(dst)
                L.w_in = dst.data_ptr()
                L.w_out = packed(p + "wd").data_ptr()
            L.wqkv = packed(p + "wqkv").data_ptr()
            L.wo = packed(p + "wo").data_ptr()
        torch.cuda.synchronize(self.device)       # packing sources may now be freed
        self._layers = layers
        mw = ModelWeights()
        emb = tok_emb if tok_emb is not None else dev(weights["tok_emb"], torch.bfloat16)
        self._keep.append(emb)
        self.tok_emb = emb                     # a draft may share this table (see tok_emb / tok_emb_stride)
        mw.tok_emb = emb.data_ptr()
        mw.tok_emb_stride = tok_emb_stride if tok_emb_stride is not None else emb.shape[1]
        mw.pos_emb = dev(weights["pos_emb"], torch.bfloat16).data_ptr() if fam_a else None
        mw.layers = layers
        mw.normf_g = dev(weights["normf_g"], torch.float32).data_ptr()
        mw.normf_b = dev(weights["normf_b"], torch.float32).data_ptr() if fam_a else None
        mw.wlm = packed("wlm").data_ptr()
        torch.cuda.synchronize(self.device)
        desc = ModelDesc(FAMILY[shape.family], shape.n_layers, shape.d_model, shape.n_heads, shape.d_head,
                         shape.n_kv_heads, shape.d_ff, shape.vocab, shape.max_pos,
                         shape.ln_eps if fam_a else shape.rms_eps, shape.rope_base)
        h = C.c_void_p()
        _check(lib().disco_model_create(C.byref(desc), C.byref(mw), C.byref(h)))
        self.handle = h

    def workspace(self, max_block: int, max_ctx: int) -> "Workspace":
        n = lib().disco_workspace_bytes(self.handle, max_block, max_ctx)
        if n == 0:
            raise DiscoError(EINVAL, "bad workspace request")
        ws = Workspace(n, self.device)
        _check(lib().disco_workspace_init(self.handle, ws.buf.data_ptr(), n, max_block, max_ctx, _stream()))
        return ws

    def prefill_workspace(self, n_tokens: int, max_ctx: int) -> "Workspace":
        """Workspace of the dense prompt pass (holds the activations of every prompt token)."""
        n = lib().disco_prefill_workspace_bytes(self.handle, n_tokens, max_ctx)
        if n == 0:
            raise DiscoError(EINVAL, "bad prefill workspace request")
        ws = Workspace(n, self.device)
        _check(lib().disco_workspace_init(self.handle, ws.buf.data_ptr(), n, MAX_BLOCK, max_ctx, _stream()))
        return ws

    def step_workspace(self, kv_prompt: "DiscoKV", seqs: "Sequences") -> "Workspace":
        """Workspace of disco_step for the prompt that kv_prompt holds now."""
        n = lib().disco_step_workspace_bytes(self.handle, kv_prompt.handle, seqs.kv.ref)
        if n == 0:
            raise DiscoError(EINVAL, last_error())
        ws = Workspace(n, self.device)
        _check(lib().disco_workspace_init(self.handle, ws.buf.data_ptr(), n, MAX_BLOCK, 0, _stream()))
        return ws

    def close(self):
        if self.handle:
            lib().disco_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Workspace:
    def __init__(self, nbytes: int, device):
        self.buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.nbytes = nbytes


class DiscoKV:
    def __init__(self, model: DiscoModel, capacity: int, page_tokens: int = 16, page_order=None):
        self.model = model
        self.capacity = -(-capacity // page_tokens) * page_tokens
        nbytes = lib().disco_kv_bytes(model.handle, capacity, page_tokens)
        self.buf = torch.empty(nbytes, dtype=torch.uint8, device=model.device)
        order = None
        if page_order is not None:
            order = (C.c_int32 * len(page_order))(*[int(p) for p in page_order])
        h = C.c_void_p()
        _check(lib().disco_kv_create(model.handle, self.buf.data_ptr(), nbytes, capacity, page_tokens,
                                     order, C.byref(h)))
        self.handle = h

    @property
    def len(self) -> int:
        return lib().disco_kv_len(self.handle)

    @property
    def pages_in_use(self) -> int:
        return lib().disco_kv_pages_in_use(self.handle)

    def fill(self, kv_tensor: torch.Tensor, stream=None):
        """kv_tensor: bf16 [n_layers, 2, ctx, n_kv_heads, d_head] on the device."""
        assert kv_tensor.dtype == torch.bfloat16 and kv_tensor.is_contiguous()
        _check(lib().disco_kv_fill(self.handle, kv_tensor.data_ptr(), kv_tensor.shape[2],
                                   _stream() if stream is None else stream))
        torch.cuda.synchronize()

    def close(self):
        if self.handle:
            lib().disco_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class DiscoClf:
    """Classifier parameters [W1 | b1 | w2 | b2] as one fp32 device vector."""

    def __init__(self, params: Dict[str, torch.Tensor], device="cuda"):
        flat = torch.cat([params["W1"].reshape(-1), params["b1"].reshape(-1), params["w2"].reshape(-1),
                          params["b2"].reshape(-1)]).to(torch.float32)
        self.dev = flat.to(device).contiguous()
        self.hidden = params["W1"].shape[0]
        self.c = Clf(self.dev.data_ptr(), self.hidden)

    def params(self) -> Dict[str, torch.Tensor]:
        """The parameter vector back as host tensors W1, b1, w2, b2."""
        h, v = self.hidden, self.dev.cpu()
        return {"W1": v[:12 * h].view(h, 12).clone(), "b1": v[12 * h:13 * h].clone(), "w2": v[13 * h:14 * h].clone(),
                "b2": v[14 * h:14 * h + 1].clone()}


def struct_tensor(ctype, n: int = 1, device="cuda", pinned: bool = False) -> torch.Tensor:
    """uint8 buffer for n records of a ctypes struct (device, or pinned host)."""
    nbytes = C.sizeof(ctype) * n
    if pinned:
        return torch.zeros(nbytes, dtype=torch.uint8, pin_memory=True)
    return torch.zeros(nbytes, dtype=torch.uint8, device=device)


def read_struct(ctype, t: torch.Tensor, index: int = 0):
    raw = bytes(t.cpu().numpy().tobytes())
    sz = C.sizeof(ctype)
    return ctype.from_buffer_copy(raw[index * sz:(index + 1) * sz])
