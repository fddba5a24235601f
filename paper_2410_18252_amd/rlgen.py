"""ctypes binding of librlgen.so: argument marshalling only.

Function names mirror include/rlgen.h.  Device buffers are torch tensors (torch is used for device
memory and streams, nothing else); every step of generation and scoring runs in the library's
kernels.  There is no fallback: if the shared library is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Dict, NamedTuple, Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librlgen.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2410_18252_amd.build`")
lib = C.CDLL(LIB_PATH)

OK = 0
ERR_NULL, ERR_BAD_CFG, ERR_BAD_ARG, ERR_CAPACITY, ERR_WORKSPACE, ERR_UNIMPLEMENTED, ERR_DEVICE = -1, -2, -3, -4, -5, -6, -7
ARCH_NEOX, ARCH_LLAMA = 0, 1
DTYPE_F32, DTYPE_BF16, DTYPE_F16, DTYPE_E4M3 = 0, 1, 2, 3

EXPORTS = ["rlgen_workspace_bytes", "rlgen_create", "rlgen_update_weights", "rlgen_generate", "rlgen_score",
           "rlgen_debug_logits", "rlgen_debug_sample", "rlgen_sample_static", "rlgen_sequence_logprob", "rlgen_dpo_loss", "rlgen_select_pairs", "rlgen_proximal_rloo",
           "rlgen_get_timings", "rlgen_set_profiling", "rlgen_set_decode_split", "rlgen_set_decode_split_min", "rlgen_set_eos",
           "rlgen_set_eos_compaction", "rlgen_set_score_groups", "rlgen_debug_get_gemm", "rlgen_debug_set_gemm", "rlgen_status",
           "rlgen_status_bits", "rlgen_strerror", "rlgen_destroy", "rlgen_plan_pages", "rlgen_rope_table", "rlgen_qk_norm_rope",
           "rlgen_qk_norm_rope_backward", "rlgen_qk_norm_rope_backward_workspace", "rlgen_window_attention",
           "rlgen_window_attention_backward", "rlgen_window_attention_backward_workspace", "rlgen_window_attention_paged",
           "rlgen_window_attention_paged_workspace", "rlgen_window_attention_chunk_workspace", "rlgen_add_rms_norm",
           "rlgen_add_rms_norm_backward", "rlgen_add_rms_norm_backward_workspace", "rlgen_token_logprobs", "rlgen_token_logprobs_workspace", "rlgen_token_logprobs_backward",
           "rlgen_dpo_pairs"]
FAULT_TOKEN, FAULT_UNIFORM, FAULT_GROUP, FAULT_RANGE = 1, 2, 4, 8
PLAN_ROWS, PLAN_PAGES, PLAN_TABLE, PLAN_LENGTH = 1, 2, 4, 8


class ModelCfg(C.Structure):
    _fields_ = [("arch", C.c_int32), ("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("d_ffn", C.c_int32), ("vocab", C.c_int32),
                ("rotary_dim", C.c_int32), ("rope_theta", C.c_float), ("norm_eps", C.c_float),
                ("weight_dtype", C.c_int32), ("max_seqs", C.c_int32), ("max_seq_len", C.c_int32),
                ("max_kv_tokens", C.c_int64), ("max_batch_tokens", C.c_int32), ("share_prompt_kv", C.c_int32),
                ("precise", C.c_int32)]


LAYER_FIELDS = ["norm1_g", "norm1_b", "norm2_g", "norm2_b", "wq", "wk", "wv", "bq", "bk", "bv", "wo", "bo",
                "w_up", "b_up", "w_gate", "w_down", "b_down"]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in LAYER_FIELDS]


class Weights(C.Structure):
    _fields_ = [("embed_in", C.c_void_p), ("final_norm_g", C.c_void_p), ("final_norm_b", C.c_void_p),
                ("lm_head", C.c_void_p), ("layers", C.POINTER(LayerWeights))]


_vp, _i32, _f32, _i64, _size = C.c_void_p, C.c_int32, C.c_float, C.c_int64, C.c_size_t
lib.rlgen_workspace_bytes.restype = C.c_size_t
lib.rlgen_workspace_bytes.argtypes = [C.POINTER(ModelCfg)]
lib.rlgen_create.restype = C.c_int
lib.rlgen_create.argtypes = [C.POINTER(ModelCfg), C.POINTER(Weights), _vp, C.c_size_t, _vp, C.POINTER(_vp)]
lib.rlgen_update_weights.restype = C.c_int
lib.rlgen_update_weights.argtypes = [_vp, C.POINTER(Weights), _vp]
lib.rlgen_generate.restype = C.c_int
lib.rlgen_generate.argtypes = [_vp, _vp, C.POINTER(_i32), _i32, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _vp, _vp]
lib.rlgen_score.restype = C.c_int
lib.rlgen_score.argtypes = [_vp, _vp, C.POINTER(_i32), C.POINTER(_i32), _i32, _i32, _f32, _vp, _vp]
lib.rlgen_debug_logits.restype = C.c_int
lib.rlgen_debug_logits.argtypes = [_vp, _vp, C.POINTER(_i32), _i32, _i32, _vp, _vp]
lib.rlgen_debug_sample.restype = C.c_int
lib.rlgen_debug_sample.argtypes = [_vp, _vp, _i32, _f32, _vp, _vp, _vp, _vp, _vp]
lib.rlgen_sample_static.restype = C.c_int
lib.rlgen_sample_static.argtypes = [_vp, _vp, _i32, _f32, _vp, _vp, _vp, _vp, _vp]
lib.rlgen_sequence_logprob.restype = C.c_int
lib.rlgen_sequence_logprob.argtypes = [_vp, _vp, _vp, _i32, _i32, _vp, _vp]
lib.rlgen_select_pairs.restype = C.c_int
lib.rlgen_select_pairs.argtypes = [_vp, _i32, _i32, _vp, _vp, _vp]
lib.rlgen_proximal_rloo.restype = C.c_int
lib.rlgen_proximal_rloo.argtypes = [_vp, _vp, _vp, _i32, _i32, _f32, _vp, _vp]
lib.rlgen_dpo_loss.restype = C.c_int
lib.rlgen_dpo_loss.argtypes = [_vp, _vp, _vp, _vp, _i32, _f32, _vp, _vp]
lib.rlgen_get_timings.restype = C.c_int
lib.rlgen_get_timings.argtypes = [_vp, C.POINTER(_f32), C.POINTER(_f32), C.POINTER(_f32), C.POINTER(_i32)]
lib.rlgen_set_score_groups.restype = C.c_int
lib.rlgen_set_score_groups.argtypes = [_vp, _i32]
lib.rlgen_set_eos.restype = C.c_int
lib.rlgen_set_eos.argtypes = [_vp, _i32]
lib.rlgen_set_decode_split.restype = C.c_int
lib.rlgen_set_decode_split.argtypes = [_vp, _i32]
lib.rlgen_set_profiling.restype = C.c_int
lib.rlgen_set_profiling.argtypes = [_vp, _i32]
lib.rlgen_status.restype = C.c_int
lib.rlgen_status.argtypes = [_vp, _vp]
lib.rlgen_status_bits.restype = C.c_int
lib.rlgen_status_bits.argtypes = [_vp, _vp, C.POINTER(C.c_uint32)]
lib.rlgen_set_eos_compaction.restype = C.c_int
lib.rlgen_set_eos_compaction.argtypes = [_vp, _i32]
lib.rlgen_set_decode_split_min.restype = C.c_int
lib.rlgen_set_decode_split_min.argtypes = [_vp, _i32]
lib.rlgen_debug_get_gemm.restype = C.c_int
lib.rlgen_debug_get_gemm.argtypes = [_vp, _i32, _i32, C.POINTER(_i32), C.POINTER(_i32)]
lib.rlgen_debug_set_gemm.restype = C.c_int
lib.rlgen_debug_set_gemm.argtypes = [_vp, _i32, _i32, _i32]
lib.rlgen_strerror.restype = C.c_char_p
lib.rlgen_strerror.argtypes = [C.c_int]
_NORM_ROPE = [_vp, _i64, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _f32, _vp, _i32, _i32, _vp, _i32]
_ROWS = [_vp, _i64]
for _name, _types in {
        "rlgen_plan_pages": [_vp, _vp, _i32, _i32, _vp, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp],
        "rlgen_rope_table": [_vp, _i32, _i32, _f32, _vp],
        "rlgen_qk_norm_rope": _NORM_ROPE + 3 * _ROWS + [_vp, _i32, _i32, _vp, _vp],
        "rlgen_qk_norm_rope_backward": _NORM_ROPE + 4 * _ROWS + [_vp, _vp, _vp, _size, _vp],
        "rlgen_window_attention": 3 * _ROWS + [_i32] * 5 + [_vp] + [_i32] * 4 + [_f32] + _ROWS + [_vp, _vp],
        "rlgen_window_attention_backward": 4 * _ROWS + [_vp] + _ROWS + [_i32] * 5 + [_vp] + [_i32] * 4 + [_f32] + 3 * _ROWS + [_vp, _size, _vp],
        "rlgen_window_attention_paged": _ROWS + [_i32] * 5 + [_vp, _i32, _i32, _vp, _i32, _vp, _vp] + [_i32] * 5 + [_f32] + _ROWS + [_vp, _vp, _size, _vp],
        "rlgen_add_rms_norm": _ROWS + [_i32] + _ROWS + [_i32] * 3 + [C.c_double, _vp, _vp, _f32] + 2 * _ROWS + [_i32, _vp, _i32, _vp],
        "rlgen_add_rms_norm_backward": _ROWS + [_i32] + _ROWS + [_i32] + _ROWS + [_i32] * 2 + [C.c_double, _vp, _vp, _f32] + 2 * _ROWS + [_vp, _vp, _size, _vp],
        "rlgen_token_logprobs": _ROWS + [_i32] * 3 + [_vp, _f32, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _size, _vp],
        "rlgen_token_logprobs_backward": _ROWS + [_i32] * 3 + [_vp, _f32, _vp, _vp, _vp, _vp] + _ROWS + [_vp],
        "rlgen_dpo_pairs": [_vp, _vp, _i32, _vp, _i32, _i32, _vp, _vp, _f32, _f32, _vp, _vp, _vp]}.items():
    getattr(lib, _name).restype, getattr(lib, _name).argtypes = C.c_int, _types
for _name, _count in {"rlgen_qk_norm_rope_backward_workspace": 2, "rlgen_window_attention_backward_workspace": 8,
                      "rlgen_window_attention_paged_workspace": 8,
                      "rlgen_window_attention_chunk_workspace": 8, "rlgen_add_rms_norm_backward_workspace": 2,
                      "rlgen_token_logprobs_workspace": 4}.items():
    getattr(lib, _name).restype, getattr(lib, _name).argtypes = _size, [_i32] * _count
lib.rlgen_destroy.restype = None
lib.rlgen_destroy.argtypes = [_vp]


class RlgenError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {rlgen_strerror(code)} ({code})")


def rlgen_strerror(code: int) -> str:
    return lib.rlgen_strerror(int(code)).decode()


def _check(code: int, where: str):
    if code != OK:
        raise RlgenError(code, where)


# plain integers (the argument types make pointers of them) and the raw stream: the objects in between cost a short call 1 to 2 us
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # not a public name: the stream object where it is missing


def _stream():
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(torch.cuda.current_device())


def _host_i32(a):
    a = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    return a, a.ctypes.data_as(C.POINTER(_i32))


def make_cfg(model, *, weight_dtype: int, max_seqs: int, max_seq_len: int, max_kv_tokens: int,
             max_batch_tokens: int = 0, share_prompt_kv: int = 0, precise: int = 0) -> ModelCfg:
    """ModelCfg from any object with the model-shape fields (arch, n_layers, d_model, ...)."""
    return ModelCfg(model.arch, model.n_layers, model.d_model, model.n_q_heads, model.n_kv_heads, model.head_dim,
                    model.d_ffn, model.vocab, model.rotary_dim, model.rope_theta, model.norm_eps, weight_dtype,
                    max_seqs, max_seq_len, max_kv_tokens, max_batch_tokens, share_prompt_kv, precise)


def rlgen_workspace_bytes(cfg: ModelCfg) -> int:
    return int(lib.rlgen_workspace_bytes(C.byref(cfg)))


def upload_weights(tensors: Dict[str, np.ndarray], device="cuda") -> Dict[str, torch.Tensor]:
    """Copies canonical tensors to the device: float32 arrays as fp32, uint16 arrays as bf16 bit patterns."""
    out = {}
    for k, v in tensors.items():
        if v.dtype == np.uint16:
            out[k] = torch.from_numpy(v.view(np.int16)).to(device).view(torch.bfloat16)
        else:
            out[k] = torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).to(device)
    return out


def _weights_struct(cfg: ModelCfg, dev: Dict[str, torch.Tensor]):
    want = torch.bfloat16 if cfg.weight_dtype == DTYPE_BF16 else torch.float32
    for k, t in dev.items():
        if t.dtype != want or not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"tensor {k}: expected contiguous device {want}")
    layers = (LayerWeights * cfg.n_layers)()
    for l in range(cfg.n_layers):
        for f in LAYER_FIELDS:
            t = dev.get(f"layers.{l}.{f}")
            setattr(layers[l], f, None if t is None else t.data_ptr())
    w = Weights(dev["embed_in"].data_ptr(), dev["final_norm_g"].data_ptr(),
                dev["final_norm_b"].data_ptr() if "final_norm_b" in dev else None, dev["lm_head"].data_ptr(), layers)
    return w, layers


class Policy:
    """Owns a context and the workspace tensor behind it."""

    def __init__(self, cfg: ModelCfg, dev_weights: Dict[str, torch.Tensor]):
        need = rlgen_workspace_bytes(cfg)
        if need == 0:
            raise RlgenError(ERR_BAD_CFG, "rlgen_workspace_bytes")
        self.cfg = cfg
        self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        w, keep = _weights_struct(cfg, dev_weights)
        ctx = C.c_void_p()
        _check(lib.rlgen_create(C.byref(cfg), C.byref(w), _ptr(self.workspace), need, _stream(), C.byref(ctx)),
               "rlgen_create")
        self.ctx = ctx
        torch.cuda.current_stream().synchronize()   # the library no longer reads dev_weights after this

    def close(self):
        if getattr(self, "ctx", None):
            lib.rlgen_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def update_weights(self, dev_weights):
        w, keep = _weights_struct(self.cfg, dev_weights)
        _check(lib.rlgen_update_weights(self.ctx, C.byref(w), _stream()), "rlgen_update_weights")
        torch.cuda.current_stream().synchronize()


def rlgen_update_weights(p: Policy, dev_weights: Dict[str, torch.Tensor]):
    p.update_weights(dev_weights)


def rlgen_generate(p: Policy, prompts: torch.Tensor, prompt_lens, k: int, max_new: int, temperature: float,
                   uniforms: torch.Tensor, forced: Optional[torch.Tensor] = None, out=None):
    """prompts int32 [B, stride] (device), prompt_lens host ints [B], uniforms fp32 [B, k, max_new] (device).
    Returns (tokens int32 [B, k, max_new], token_logprobs fp32 [B, k, max_new]) on the device; asynchronous."""
    B, stride = prompts.shape
    assert prompts.dtype == torch.int32 and prompts.is_contiguous() and prompts.is_cuda
    assert uniforms.dtype == torch.float32 and uniforms.is_contiguous() and tuple(uniforms.shape) == (B, k, max_new)
    if forced is not None:
        assert forced.dtype == torch.int32 and forced.is_contiguous() and tuple(forced.shape) == (B, k, max_new)
    lens, lens_p = _host_i32(prompt_lens)
    assert lens.shape == (B,)
    if out is None:
        tokens = torch.empty((B, k, max_new), dtype=torch.int32, device=prompts.device)
        lps = torch.empty((B, k, max_new), dtype=torch.float32, device=prompts.device)
    else:
        tokens, lps = out
    _check(lib.rlgen_generate(p.ctx, _ptr(prompts), lens_p, B, stride, k, max_new, temperature, _ptr(uniforms),
                              _ptr(forced), _ptr(tokens), _ptr(lps), _stream()), "rlgen_generate")
    return tokens, lps


def rlgen_score(p: Policy, seqs: torch.Tensor, seq_lens, temperature: float, score_from=None, out=None):
    N, stride = seqs.shape
    assert seqs.dtype == torch.int32 and seqs.is_contiguous() and seqs.is_cuda
    lens, lens_p = _host_i32(seq_lens)
    assert lens.shape == (N,)
    sf, sf_p = (None, None) if score_from is None else _host_i32(score_from)
    lps = torch.empty((N, stride), dtype=torch.float32, device=seqs.device) if out is None else out
    _check(lib.rlgen_score(p.ctx, _ptr(seqs), lens_p, sf_p, N, stride, temperature, _ptr(lps), _stream()), "rlgen_score")
    return lps


def rlgen_debug_logits(p: Policy, seqs: torch.Tensor, seq_lens):
    N, stride = seqs.shape
    assert seqs.dtype == torch.int32 and seqs.is_contiguous() and seqs.is_cuda
    lens, lens_p = _host_i32(seq_lens)
    logits = torch.empty((N, p.cfg.vocab), dtype=torch.float32, device=seqs.device)
    _check(lib.rlgen_debug_logits(p.ctx, _ptr(seqs), lens_p, N, stride, _ptr(logits), _stream()), "rlgen_debug_logits")
    return logits


def rlgen_debug_sample(p: Policy, hidden: torch.Tensor, temperature: float, uniforms: torch.Tensor,
                       forced: Optional[torch.Tensor] = None):
    R, d = hidden.shape
    assert hidden.dtype == torch.float32 and hidden.is_contiguous() and d == p.cfg.d_model
    assert uniforms.dtype == torch.float32 and tuple(uniforms.shape) == (R,)
    tokens = torch.empty(R, dtype=torch.int32, device=hidden.device)
    lps = torch.empty(R, dtype=torch.float32, device=hidden.device)
    _check(lib.rlgen_debug_sample(p.ctx, _ptr(hidden), R, temperature, _ptr(uniforms), _ptr(forced), _ptr(tokens),
                                  _ptr(lps), _stream()), "rlgen_debug_sample")
    return tokens, lps


def rlgen_sample_static(p: Policy, hidden: torch.Tensor, temperature: float, uniforms: torch.Tensor,
                        forced: Optional[torch.Tensor] = None, out=None):
    """rlgen_debug_sample with the library's static scratch; `out` = (tokens, token_logprobs) to write into."""
    R, d = hidden.shape
    assert hidden.dtype == torch.float32 and hidden.is_contiguous() and d == p.cfg.d_model
    assert uniforms.dtype == torch.float32 and tuple(uniforms.shape) == (R,)
    tokens, lps = out if out is not None else (torch.empty(R, dtype=torch.int32, device=hidden.device),
                                               torch.empty(R, dtype=torch.float32, device=hidden.device))
    _check(lib.rlgen_sample_static(p.ctx, _ptr(hidden), R, temperature, _ptr(uniforms), _ptr(forced), _ptr(tokens),
                                   _ptr(lps), _stream()), "rlgen_sample_static")
    return tokens, lps


def rlgen_sequence_logprob(token_logprobs: torch.Tensor, start: torch.Tensor, lens: torch.Tensor):
    N, stride = token_logprobs.shape
    assert token_logprobs.dtype == torch.float32 and token_logprobs.is_contiguous()
    assert start.dtype == torch.int32 and lens.dtype == torch.int32
    out = token_logprobs.new_empty(N)
    _check(lib.rlgen_sequence_logprob(_ptr(token_logprobs), _ptr(start), _ptr(lens), N, stride, _ptr(out), _stream()),
           "rlgen_sequence_logprob")
    return out


def rlgen_dpo_loss(pol_pos, ref_pos, pol_neg, ref_neg, beta: float):
    P = pol_pos.numel()
    for t in (pol_pos, ref_pos, pol_neg, ref_neg):
        assert t.dtype == torch.float32 and t.is_contiguous() and t.numel() == P
    out = pol_pos.new_empty(P)
    _check(lib.rlgen_dpo_loss(_ptr(pol_pos), _ptr(ref_pos), _ptr(pol_neg), _ptr(ref_neg), P, beta, _ptr(out), _stream()),
           "rlgen_dpo_loss")
    return out


def rlgen_proximal_rloo(pol_logprob, old_logprob, rewards, epsilon: float):
    """[B, k] fp32 sequence log-probs under pi_theta and pi_old and rewards -> [B, k] clipped objective."""
    assert rewards.dim() == 2
    B, k = rewards.shape
    for t in (pol_logprob, old_logprob, rewards):
        assert t.dtype == torch.float32 and t.is_contiguous() and tuple(t.shape) == (B, k)
    out = rewards.new_empty((B, k))
    _check(lib.rlgen_proximal_rloo(_ptr(pol_logprob), _ptr(old_logprob), _ptr(rewards), B, k, epsilon, _ptr(out), _stream()),
           "rlgen_proximal_rloo")
    return out


def rlgen_select_pairs(rewards):
    """rewards [B, k] fp32 on the device -> (idx_pos, idx_neg), each [B] int32."""
    assert rewards.dtype == torch.float32 and rewards.is_contiguous() and rewards.dim() == 2
    B, k = rewards.shape
    pos, neg = rewards.new_empty(B, dtype=torch.int32), rewards.new_empty(B, dtype=torch.int32)
    _check(lib.rlgen_select_pairs(_ptr(rewards), B, k, _ptr(pos), _ptr(neg), _stream()), "rlgen_select_pairs")
    return pos, neg


def rlgen_get_timings(p: Policy):
    a, b, c, n = _f32(), _f32(), _f32(), _i32()
    _check(lib.rlgen_get_timings(p.ctx, C.byref(a), C.byref(b), C.byref(c), C.byref(n)), "rlgen_get_timings")
    return {"prefill_ms": a.value, "decode_ms": b.value, "decode_attn_ms": c.value, "decode_attn_launches": n.value}


def rlgen_set_score_groups(p: Policy, k: int):
    _check(lib.rlgen_set_score_groups(p.ctx, int(k)), "rlgen_set_score_groups")


def rlgen_set_eos(p: Policy, eos_token: int):
    _check(lib.rlgen_set_eos(p.ctx, int(eos_token)), "rlgen_set_eos")


def rlgen_set_decode_split(p: Policy, on: bool):
    _check(lib.rlgen_set_decode_split(p.ctx, 1 if on else 0), "rlgen_set_decode_split")


def rlgen_set_profiling(p: Policy, every: int):
    """every >= 1: bracket every `every`-th decode-attention launch with events; 0 / False: off."""
    _check(lib.rlgen_set_profiling(p.ctx, int(every)), "rlgen_set_profiling")


def rlgen_status(p: Policy) -> int:
    return int(lib.rlgen_status(p.ctx, _stream()))


def rlgen_status_bits(p: Policy) -> int:
    """The sticky fault bits (FAULT_*); synchronises the current stream."""
    bits = C.c_uint32()
    lib.rlgen_status_bits(p.ctx, _stream(), C.byref(bits))
    return int(bits.value)


def rlgen_set_eos_compaction(p: Policy, every: int):
    _check(lib.rlgen_set_eos_compaction(p.ctx, int(every)), "rlgen_set_eos_compaction")


def rlgen_set_decode_split_min(p: Policy, min_seqs: int):
    _check(lib.rlgen_set_decode_split_min(p.ctx, int(min_seqs)), "rlgen_set_decode_split_min")


def rlgen_debug_get_gemm(p: Policy, mode: int, which: int):
    """(tile-shape variant, K split) of linear layer `which` in `mode`."""
    v, sp = _i32(), _i32()
    _check(lib.rlgen_debug_get_gemm(p.ctx, mode, which, C.byref(v), C.byref(sp)), "rlgen_debug_get_gemm")
    return v.value, sp.value


def rlgen_debug_set_gemm(p: Policy, mode: int, which: int, variant: int):
    _check(lib.rlgen_debug_set_gemm(p.ctx, mode, which, int(variant)), "rlgen_debug_set_gemm")


# ------------------------------------------------------------------ operators over a cache in pages and packed rows
# They stand outside autograd: outputs carry no history whatever their inputs ask for, gradients come from the *_backward functions.
_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}


_I32, _F32 = torch.int32, torch.float32


def _heads(t: torch.Tensor, dtype: torch.dtype):
    """[rows, heads, head_dim] with heads and head_dim contiguous: (address, row stride)."""
    rows, heads, h = t.shape
    row, head, dim = t.stride()
    assert t.dtype is dtype and t.is_cuda and dim == 1 and (head == h or heads == 1)
    # (the row stride of a tensor of one row or none means nothing)
    return t.data_ptr(), row if rows > 1 else heads * h


def _ints(t: torch.Tensor, *shape):
    assert t.dtype is _I32 and t.is_cuda and t.shape == shape and t.is_contiguous()
    return t.data_ptr()


def _floats(t: torch.Tensor, n: int):
    assert t.dtype is _F32 and t.is_cuda and t.numel() == n and t.is_contiguous()
    return t.data_ptr()


def _space(t: Optional[torch.Tensor]):
    """A workspace's address and bytes."""
    if t is None:
        return None, 0
    assert t.is_cuda and t.is_contiguous()
    return t.data_ptr(), t.numel() * t.element_size()


class PagePlan(NamedTuple):
    """What rlgen_plan_pages fills, all int32 on the device: total_lens [S], row_starts [S + 1], slots and positions [max_rows],
    counts [4] (rows, the free list's next head, longest length, PLAN_* bits)."""
    total_lens: torch.Tensor
    row_starts: torch.Tensor
    slots: torch.Tensor
    positions: torch.Tensor
    counts: torch.Tensor


def rlgen_plan_pages(ctx_lens: torch.Tensor, new_lens: torch.Tensor, page_size: int, free_pages: torch.Tensor, page_table: torch.Tensor,
                     max_rows: int, free_head: Optional[torch.Tensor] = None, out=None) -> PagePlan:
    """ctx_lens, new_lens [S], free_pages [n], page_table [S, pages of a sequence] (in and out), free_head [1] or None: int32 on the
    device.  `out`: a PagePlan (or tuple) of tensors to fill."""
    S, stride = page_table.shape
    if out is None:
        buf = ctx_lens.new_empty(2 * S + 5 + 2 * max_rows)
        out = torch.split(buf, [S, S + 1, max_rows, max_rows, 4])
    total_lens, row_starts, slots, positions, counts = out
    n_free = free_pages.numel()
    _check(lib.rlgen_plan_pages(_ints(ctx_lens, S), _ints(new_lens, S), S, page_size, _ints(free_pages, n_free), n_free,
                                None if free_head is None else _ints(free_head, 1), _ints(page_table, S, stride), stride, max_rows,
                                _ints(total_lens, S), _ints(row_starts, S + 1), _ints(slots, max_rows), _ints(positions, max_rows),
                                _ints(counts, 4), _stream()), "rlgen_plan_pages")
    return out if type(out) is PagePlan else PagePlan(total_lens, row_starts, slots, positions, counts)


def rlgen_rope_table(max_pos: int, rotary_dim: int, theta: float, device="cuda") -> torch.Tensor:
    """[max_pos, rotary_dim / 2, 2] fp32: cos and sin."""
    table = torch.empty((max_pos, rotary_dim // 2, 2), dtype=torch.float32, device=device)
    _check(lib.rlgen_rope_table(_floats(table, table.numel()), max_pos, rotary_dim, theta, _stream()), "rlgen_rope_table")
    return table


def _norm_rope_args(qkv, q_gain, k_gain, eps, rope, positions, n_q, n_kv, dtype):
    rows, width = qkv.shape
    row, dim = qkv.stride()
    h = q_gain.numel()
    assert qkv.is_cuda and dim == 1 and width == (n_q + 2 * n_kv) * h
    assert q_gain.dtype is _F32 and q_gain.is_cuda and q_gain.is_contiguous()
    assert k_gain.dtype is _F32 and k_gain.is_cuda and k_gain.is_contiguous() and k_gain.numel() == h
    max_pos, half = 1, 0
    if rope is not None:
        max_pos, half, two = rope.shape
        assert rope.dtype is _F32 and rope.is_cuda and rope.is_contiguous() and two == 2
    return (qkv.data_ptr(), row if rows > 1 else width, _DTYPES[qkv.dtype], rows, n_q, n_kv, h, q_gain.data_ptr(), k_gain.data_ptr(), eps,
            None if rope is None else rope.data_ptr(), max_pos, 2 * half, _ints(positions, rows), _DTYPES[dtype])


def _pages(pages: torch.Tensor, n_kv: int, h: int):
    n_pages, two, heads, page_size, dims = pages.shape
    assert pages.is_cuda and pages.is_contiguous() and two == 2 and heads == n_kv and dims == h
    return pages.data_ptr(), n_pages, page_size


def rlgen_qk_norm_rope(qkv: torch.Tensor, q_gain: torch.Tensor, k_gain: torch.Tensor, eps: float, rope: Optional[torch.Tensor],
                       positions: torch.Tensor, pages: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                       n_kv_heads: Optional[int] = None, dtype: Optional[torch.dtype] = None, out=None):
    """qkv [rows, (n_q + 2 n_kv) h] (fp32, bf16 or fp16; any row stride) -> q [rows, n_q, h].  With `pages` [n, 2, n_kv, page_size, h] keys and
    values go to slots [rows] of them and q is returned; without, n_kv_heads says how many there are and (q, k, v) of `dtype` (default
    qkv's) are returned.  `out`: q, or (q, k, v), to write into."""
    h = q_gain.numel()
    n_kv = pages.shape[2] if pages is not None else n_kv_heads
    n_q = qkv.shape[1] // h - 2 * n_kv
    rows = qkv.shape[0]
    if pages is not None:
        dtype = pages.dtype
        q, k, v = (torch.empty((rows, n_q, h), dtype=dtype, device=qkv.device) if out is None else out), None, None
        where = (*_pages(pages, n_kv, h), _ints(slots, rows))
        rest = (None, 0, None, 0)
    else:
        dtype = qkv.dtype if dtype is None else dtype
        q, k, v = out if out is not None else (torch.empty((rows, n, h), dtype=dtype, device=qkv.device) for n in (n_q, n_kv, n_kv))
        assert k.shape == v.shape == (rows, n_kv, h)
        where = (None, 0, 0, None)
        rest = (*_heads(k, dtype), *_heads(v, dtype))
    assert q.shape == (rows, n_q, h)
    _check(lib.rlgen_qk_norm_rope(*_norm_rope_args(qkv, q_gain, k_gain, eps, rope, positions, n_q, n_kv, dtype), *_heads(q, dtype), *rest, *where,
                                  _stream()), "rlgen_qk_norm_rope")
    return q if pages is not None else (q, k, v)


def rlgen_qk_norm_rope_backward(qkv, q_gain, k_gain, eps: float, rope, positions, dq, dk, dv, out=None, workspace=None):
    """dq [rows, n_q, h], dk and dv [rows, n_kv, h] -> (dqkv like qkv, dq_gain [h], dk_gain [h])."""
    rows, n_q, h = dq.shape
    n_kv = dk.shape[1]
    assert dk.shape == dv.shape == (rows, n_kv, h)
    if out is None:
        out = (torch.empty((rows, qkv.shape[1]), dtype=qkv.dtype, device=qkv.device), torch.empty_like(q_gain), torch.empty_like(k_gain))
    dqkv, dqg, dkg = out
    assert dqkv.dtype == qkv.dtype and dqkv.is_cuda and dqkv.shape == qkv.shape and dqkv.stride(1) == 1
    need = lib.rlgen_qk_norm_rope_backward_workspace(rows, h)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=qkv.device)
    _check(lib.rlgen_qk_norm_rope_backward(*_norm_rope_args(qkv, q_gain, k_gain, eps, rope, positions, n_q, n_kv, dq.dtype), *_heads(dq, dq.dtype),
                                           *_heads(dk, dq.dtype), *_heads(dv, dq.dtype), dqkv.data_ptr(), dqkv.stride(0) if rows > 1 else dqkv.shape[1],
                                           _floats(dqg, h), _floats(dkg, h), *_space(workspace), _stream()),
           "rlgen_qk_norm_rope_backward")
    return dqkv, dqg, dkg


def rlgen_window_attention(q, k, v, row_starts, max_len: int, window: int, sinks: int, scale: float, out=None):
    """Packed rows: q [rows, n_q, h], k and v [rows, n_kv, h] (any row stride), row_starts [S + 1] int32.  Returns (out [rows, n_q, h],
    lse [rows, n_q] fp32); `out`: the two to write into.  Rows that no sequence has within max_len are not written."""
    rows, n_q, h = q.shape
    n_kv, dt = k.shape[1], q.dtype
    assert k.shape == v.shape == (rows, n_kv, h)
    o, lse = out if out is not None else (torch.empty((rows, n_q, h), dtype=dt, device=q.device),
                                          torch.empty((rows, n_q), dtype=torch.float32, device=q.device))
    assert o.shape == q.shape and lse.shape == (rows, n_q)
    S = row_starts.numel() - 1
    _check(lib.rlgen_window_attention(*_heads(q, dt), *_heads(k, dt), *_heads(v, dt), _DTYPES[dt], rows, n_q, n_kv, h, _ints(row_starts, S + 1), S,
                                      max_len, window, sinks, scale, *_heads(o, dt), _floats(lse, rows * n_q), _stream()), "rlgen_window_attention")
    return o, lse


def rlgen_window_attention_backward(q, k, v, out, lse, dout, row_starts, max_len: int, window: int, sinks: int, scale: float, grads=None,
                                    workspace=None):
    """From rlgen_window_attention's inputs, its (out, lse) and dout: (dq, dk, dv).  `grads`: the three to write into.  Rows that no sequence has
    within max_len are not written."""
    rows, n_q, h = q.shape
    n_kv, dt = k.shape[1], q.dtype
    assert k.shape == v.shape == (rows, n_kv, h) and out.shape == dout.shape == q.shape and lse.shape == (rows, n_q)
    dq, dk, dv = grads if grads is not None else (torch.empty((rows, n, h), dtype=dt, device=q.device) for n in (n_q, n_kv, n_kv))
    assert dq.shape == q.shape and dk.shape == dv.shape == k.shape
    S = row_starts.numel() - 1
    need = lib.rlgen_window_attention_backward_workspace(rows, n_q, n_kv, h, S, max_len, window, sinks)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    _check(lib.rlgen_window_attention_backward(*_heads(q, dt), *_heads(k, dt), *_heads(v, dt), *_heads(out, dt), _floats(lse, rows * n_q),
                                               *_heads(dout, dt), _DTYPES[dt], rows, n_q, n_kv, h, _ints(row_starts, S + 1), S, max_len, window, sinks, scale,
                                               *_heads(dq, dt), *_heads(dk, dt), *_heads(dv, dt), *_space(workspace), _stream()),
           "rlgen_window_attention_backward")
    return dq, dk, dv


def rlgen_window_attention_paged(q, pages, page_table, row_starts, total_lens, max_new: int, max_total: int, window: int, sinks: int,
                                 scale: float, out=None, workspace=None):
    """q [rows, n_q, h]: the last row_starts[s + 1] - row_starts[s] of the total_lens[s] tokens that the cache holds of each sequence.
    Returns (out [rows, n_q, h], lse [rows, n_q] fp32); max_new == 1 is a decode step."""
    rows, n_q, h = q.shape
    n_kv, dt = pages.shape[2], q.dtype
    assert pages.dtype == dt
    S, stride = page_table.shape
    o, lse = out if out is not None else (torch.empty((rows, n_q, h), dtype=dt, device=q.device),
                                          torch.empty((rows, n_q), dtype=torch.float32, device=q.device))
    assert o.shape == q.shape and lse.shape == (rows, n_q)
    size = lib.rlgen_window_attention_paged_workspace if max_new == 1 else lib.rlgen_window_attention_chunk_workspace
    need = size(n_q, n_kv, h, S, max_new, max_total, window, sinks)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    _check(lib.rlgen_window_attention_paged(*_heads(q, dt), _DTYPES[dt], rows, n_q, n_kv, h, *_pages(pages, n_kv, h), _ints(page_table, S, stride), stride,
                                            _ints(row_starts, S + 1), _ints(total_lens, S), S, max_new, max_total, window, sinks, scale,
                                            *_heads(o, dt), _floats(lse, rows * n_q), *_space(workspace), _stream()),
           "rlgen_window_attention_paged")
    return o, lse


# ------------------------------------------------------------------ the learner's rows: norm, log-probs, loss
# They stand outside autograd too.
_E4M3 = torch.float8_e4m3fn
_NORM_DTYPES = {**_DTYPES, _E4M3: DTYPE_E4M3}


_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)       # (the former without its check for a first use: there are tensors)


def _here():
    """The current device, on which every tensor has to be, and its current stream."""
    device = _device()
    return device, torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(device)


def _rows(t: Optional[torch.Tensor], dtype: torch.dtype, shape, device: int):
    """[rows, width] with contiguous rows: (address, row stride)."""
    rows, width = shape
    if t is None:
        return None, width
    row, one = t.stride()
    assert t.dtype is dtype and t.get_device() == device and t.shape == shape and (one == 1 or width == 1)
    return t.data_ptr(), row if rows > 1 else width


def _numbers(t: Optional[torch.Tensor], dtype: torch.dtype, shape, device: int):
    """A contiguous tensor of a shape: its address."""
    if t is None:
        return None
    assert t.dtype is dtype and t.get_device() == device and t.shape == shape and t.is_contiguous()
    return t.data_ptr()


# bytes by sizes alone: a lookup instead of a call
_norm_backward_bytes = functools.lru_cache(256)(lib.rlgen_add_rms_norm_backward_workspace)
_logprobs_bytes = functools.lru_cache(256)(lib.rlgen_token_logprobs_workspace)


_MOST_INT = 2 ** 31 - 1      # (ctypes keeps the low 32 bits of what is larger)


def _scratch(t: Optional[torch.Tensor], device: int):
    if t is None:
        return None, 0
    assert t.get_device() == device and t.is_contiguous()
    return t.data_ptr(), t.numel() * t.element_size()


def rlgen_add_rms_norm(x: torch.Tensor, gain: Optional[torch.Tensor], eps: float, residual: Optional[torch.Tensor] = None, drop_p: float = 0.0,
                       rng: Optional[torch.Tensor] = None, h_dtype: Optional[torch.dtype] = None, y_dtype: Optional[torch.dtype] = None,
                       scale_group: int = 0, out=None):
    """h = residual + dropout(x) [rows, width] (residual's type; without a residual h_dtype, default x's) and y = its RMS norm times gain (fp32 [width]) of
    y_dtype (default x's; torch.float8_e4m3fn: with scales, one for scale_group columns, 0: for the row).  Returns (h, y), or (h, y, scales) for 8
    bits; gain None: y is None.  rng [2] int64: seed and offset.  `out`: what to write into, h or y None where it is not wanted.  Without
    `out`, and with nothing to add, drop or round, h is x itself."""
    shape = rows, width = x.shape
    assert rows <= _MOST_INT and width <= _MOST_INT and abs(scale_group) <= _MOST_INT
    res = residual.dtype if residual is not None else x.dtype if h_dtype is None else h_dtype
    if out is None:
        same = residual is None and drop_p == 0 and res is x.dtype
        h = None if same else torch.empty(shape, dtype=res, device=x.device)
        y = None if gain is None else torch.empty(shape, dtype=x.dtype if y_dtype is None else y_dtype, device=x.device)
        if same and y is None:
            return x, None
        out = (x if same else h, y)
        if y is not None and y.dtype is _E4M3:
            out += (torch.empty((rows, -(-width // scale_group) if scale_group > 0 else 1), dtype=_F32, device=x.device),)
    else:
        h, y = out[0], out[1]
        if h is not None and residual is None:
            res = h.dtype
    dev, stream = _here()
    scales = _numbers(out[2], _F32, (rows, -(-width // scale_group) if scale_group > 0 else 1), dev) if y is not None and y.dtype is _E4M3 else None
    ydt = x.dtype if y is None else y.dtype
    _check(lib.rlgen_add_rms_norm(*_rows(x, x.dtype, shape, dev), _DTYPES[x.dtype], *_rows(residual, res, shape, dev), _DTYPES[res], rows, width, drop_p,
                                  _numbers(rng, torch.int64, (2,), dev), _numbers(gain, _F32, (width,), dev), eps, *_rows(h, res, shape, dev),
                                  *_rows(y, ydt, shape, dev), _NORM_DTYPES[ydt], scales, scale_group, stream), "rlgen_add_rms_norm")
    return out


def rlgen_add_rms_norm_backward(h: Optional[torch.Tensor], gain: Optional[torch.Tensor], eps: float, dy: Optional[torch.Tensor],
                                dh: Optional[torch.Tensor] = None, drop_p: float = 0.0, rng: Optional[torch.Tensor] = None,
                                dtype: Optional[torch.dtype] = None, out=None, workspace=None):
    """From rlgen_add_rms_norm's h, dy (gradient of y) and dh (of h, or None): (dresidual like h, dx of x's type, dgain fp32 [width]).  x's type is
    dy's, or `dtype` where there was no norm (gain, h and dy None; dgain is None then).  `out`: the three to write into, dresidual or dx None
    where it is not wanted; without it, and with nothing dropped or rounded, dx is dresidual itself."""
    like = h if h is not None else dh
    shape = rows, width = like.shape
    assert rows <= _MOST_INT and width <= _MOST_INT
    res = like.dtype
    dt = dy.dtype if dy is not None else res if dtype is None else dtype
    if out is None:
        dres = torch.empty(shape, dtype=res, device=like.device)
        dx = None if drop_p == 0 and dt is res else torch.empty(shape, dtype=dt, device=like.device)
        dgain = None if gain is None else torch.empty(width, dtype=_F32, device=like.device)
        out = (dres, dres if dx is None else dx, dgain)
    else:
        dres, dx, dgain = out
    if gain is not None and workspace is None and (need := _norm_backward_bytes(rows, width)):
        workspace = like.new_empty(need, dtype=torch.uint8)
    dev, stream = _here()
    _check(lib.rlgen_add_rms_norm_backward(*_rows(h, res, shape, dev), _DTYPES[res], *_rows(dy, dt, shape, dev), _DTYPES[dt], *_rows(dh, res, shape, dev),
                                           rows, width, drop_p, _numbers(rng, torch.int64, (2,), dev), _numbers(gain, _F32, (width,), dev), eps,
                                           *_rows(dres, res, shape, dev), *_rows(dx, dt, shape, dev), _numbers(dgain, _F32, (width,), dev),
                                           *_scratch(workspace, dev), stream), "rlgen_add_rms_norm_backward")
    return out


class TokenLogprobs(NamedTuple):
    """What rlgen_token_logprobs fills: logprobs [rows], entropy [rows], stats [rows, 2] fp32, top_tokens [rows, n] int32, top_logprobs
    [rows, n] fp32; None where it was not asked for."""
    logprobs: Optional[torch.Tensor]
    entropy: Optional[torch.Tensor]
    stats: torch.Tensor
    top_tokens: Optional[torch.Tensor]
    top_logprobs: Optional[torch.Tensor]


def rlgen_token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, temperature: float = 1.0, entropy: bool = True, n_top: int = 0,
                         out=None, workspace=None) -> TokenLogprobs:
    """logits [rows, vocab] (fp32, bf16 or fp16; any row stride), tokens [rows] int32 or None.  A row whose token lies outside the vocabulary is skipped.
    `out`: a TokenLogprobs (or tuple) of tensors to fill; entropy and n_top are then what it holds."""
    shape = rows, vocab = logits.shape
    assert rows <= _MOST_INT and vocab <= _MOST_INT
    dev, stream = _here()
    if out is None:
        new = logits.new_empty
        lp, ent, stats = None if tokens is None else new(rows, dtype=_F32), new(rows, dtype=_F32) if entropy else None, new((rows, 2), dtype=_F32)
        ids, top = (new((rows, n_top), dtype=_I32), new((rows, n_top), dtype=_F32)) if n_top else (None, None)
        out = TokenLogprobs(lp, ent, stats, ids, top)
        where = (None if lp is None else lp.data_ptr(), stats.data_ptr(), None if ent is None else ent.data_ptr(), n_top,
                 None if ids is None else ids.data_ptr(), None if top is None else top.data_ptr())
    else:
        lp, ent, stats, ids, top = out
        n_top = 0 if ids is None else ids.shape[1]
        assert (top is None) == (ids is None) and n_top <= _MOST_INT
        where = (_numbers(lp, _F32, (rows,), dev), _numbers(stats, _F32, (rows, 2), dev), _numbers(ent, _F32, (rows,), dev), n_top,
                 _numbers(ids, _I32, (rows, n_top), dev), _numbers(top, _F32, (rows, n_top), dev))
    dt = _DTYPES[logits.dtype]
    if workspace is None and (need := _logprobs_bytes(dt, rows, vocab, n_top)):
        workspace = logits.new_empty(need, dtype=torch.uint8)
    _check(lib.rlgen_token_logprobs(*_rows(logits, logits.dtype, shape, dev), dt, rows, vocab, _numbers(tokens, _I32, (rows,), dev), temperature, *where,
                                    *_scratch(workspace, dev), stream), "rlgen_token_logprobs")
    return out if type(out) is TokenLogprobs else TokenLogprobs(lp, ent, stats, ids, top)


def rlgen_token_logprobs_backward(logits: torch.Tensor, tokens: Optional[torch.Tensor], temperature: float, stats: torch.Tensor,
                                  dlogprobs: Optional[torch.Tensor], entropy: Optional[torch.Tensor] = None, dentropy: Optional[torch.Tensor] = None,
                                  out=None):
    """From rlgen_token_logprobs's inputs, its stats (and entropy, with dentropy) and the gradients [rows] of logprobs and entropy: dlogits like
    logits.  `out` may be logits itself."""
    shape = rows, vocab = logits.shape
    assert rows <= _MOST_INT and vocab <= _MOST_INT
    if out is None:
        out = torch.empty(shape, dtype=logits.dtype, device=logits.device)
    dev, stream = _here()
    _check(lib.rlgen_token_logprobs_backward(*_rows(logits, logits.dtype, shape, dev), _DTYPES[logits.dtype], rows, vocab, _numbers(tokens, _I32, (rows,), dev),
                                             temperature, _numbers(stats, _F32, (rows, 2), dev), _numbers(entropy, _F32, (rows,), dev),
                                             _numbers(dlogprobs, _F32, (rows,), dev), _numbers(dentropy, _F32, (rows,), dev),
                                             *_rows(out, logits.dtype, shape, dev), stream), "rlgen_token_logprobs_backward")
    return out


def rlgen_dpo_pairs(token_logprobs: torch.Tensor, ref_logprobs: torch.Tensor, row_starts: torch.Tensor, idx_pos: torch.Tensor, idx_neg: torch.Tensor,
                    k: int, beta: float, weight: float = 1.0, out=None):
    """token_logprobs, ref_logprobs [rows] fp32 of packed sequences, row_starts [B k + 1], idx_pos and idx_neg [B] int32.  Returns (loss [B], the gradient
    of weight times the losses' sum to token_logprobs [rows]).  Rows that no sequence has are 0; with `out`, the two to write into, they are left as they
    are, and the launch that zeroes them falls away."""
    rows, B = token_logprobs.numel(), idx_pos.numel()
    assert rows <= _MOST_INT and B <= _MOST_INT and abs(k) <= _MOST_INT
    loss, grad = out if out is not None else (token_logprobs.new_empty(B), token_logprobs.new_zeros(rows))
    dev, stream = _here()
    _check(lib.rlgen_dpo_pairs(_numbers(token_logprobs, _F32, (rows,), dev), _numbers(ref_logprobs, _F32, (rows,), dev), rows,
                               _numbers(row_starts, _I32, (B * k + 1,), dev), B, k, _numbers(idx_pos, _I32, (B,), dev), _numbers(idx_neg, _I32, (B,), dev), beta,
                               weight, _numbers(loss, _F32, (B,), dev), _numbers(grad, _F32, (rows,), dev), stream), "rlgen_dpo_pairs")
    return loss, grad
