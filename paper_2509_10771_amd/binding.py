"""ctypes binding with the same names as the C ABI in include/rslx.h (argument marshalling only)."""
import ctypes as C
import os

import torch

__all__ = [
    "RslxError", "lib", "Mlp", "Rollout", "PpoCfg", "BcCfg", "Sym", "RndTrain", "workspace", "NSTATS",
    "rslx_version", "rslx_device_check", "rslx_permutation", "rslx_permutation_workspace_bytes",
    "rslx_act", "rslx_act_workspace_bytes", "rslx_gae", "rslx_gae_workspace_bytes",
    "rslx_adam_step", "rslx_adam_workspace_bytes", "rslx_ppo_update", "rslx_ppo_update_workspace_bytes",
    "rslx_bc_update", "rslx_bc_update_workspace_bytes", "rslx_sym_augment", "rslx_rnd", "rslx_rnd_workspace_bytes",
    "ACT_DETERMINISTIC", "ACT_VALUES_ONLY", "EXPORTS", "rslx_trace_begin", "rslx_trace_end",
    "dev_counters", "rslx_act_dc", "rslx_ppo_update_dc", "rslx_bc_update_dc", "rslx_bc_collect_workspace_bytes",
    "rslx_bc_collect", "Memory", "Gru", "Lstm", "CELL_GRU", "CELL_LSTM", "rslx_act_recurrent_workspace_bytes", "rslx_act_recurrent",
    "rslx_ppo_update_recurrent_workspace_bytes", "rslx_ppo_update_recurrent", "rslx_memory_step_workspace_bytes",
    "rslx_memory_step", "rslx_bc_update_recurrent_workspace_bytes", "rslx_bc_update_recurrent",
    "rslx_act_recurrent_dc", "rslx_ppo_update_recurrent_dc", "rslx_gae_noalloc", "GAE_NOALLOC_MAX_ENVS",
    "LinearAttn", "ATTN_MAX_DIM", "NORM_MAX_COLS", "rslx_linear_attention_workspace_bytes", "rslx_linear_attention",
    "rslx_linear_attention_backward_workspace_bytes", "rslx_linear_attention_backward", "rslx_linear_attention_step",
    "rslx_layer_norm", "rslx_layer_norm_backward_workspace_bytes", "rslx_layer_norm_backward",
    "GatedRec", "Muon", "rslx_gated_recurrence_workspace_bytes", "rslx_gated_recurrence",
    "rslx_gated_recurrence_backward_workspace_bytes", "rslx_gated_recurrence_backward", "rslx_gated_recurrence_step",
    "rslx_rms_norm", "rslx_rms_norm_e4m3", "rslx_rms_norm_backward_workspace_bytes", "rslx_rms_norm_backward",
    "rslx_muon_step_workspace_bytes", "rslx_muon_step",
]

MAX_LAYERS = 8
NSTATS = 8
ACT_DETERMINISTIC = 1
ACT_VALUES_ONLY = 2

EXPORTS = [
    "rslx_version", "rslx_last_error", "rslx_device_check", "rslx_permutation_workspace_bytes", "rslx_permutation",
    "rslx_act_workspace_bytes", "rslx_act", "rslx_gae_workspace_bytes", "rslx_gae", "rslx_adam_workspace_bytes",
    "rslx_adam_step", "rslx_ppo_update_workspace_bytes", "rslx_ppo_update", "rslx_bc_update_workspace_bytes",
    "rslx_bc_update", "rslx_sym_augment", "rslx_rnd_workspace_bytes", "rslx_rnd", "rslx_trace_begin", "rslx_trace_end",
    "rslx_act_dc", "rslx_ppo_update_dc", "rslx_bc_update_dc", "rslx_bc_collect_workspace_bytes", "rslx_bc_collect",
    "rslx_act_recurrent_workspace_bytes", "rslx_act_recurrent", "rslx_ppo_update_recurrent_workspace_bytes",
    "rslx_ppo_update_recurrent", "rslx_memory_step_workspace_bytes", "rslx_memory_step",
    "rslx_bc_update_recurrent_workspace_bytes", "rslx_bc_update_recurrent", "rslx_act_recurrent_dc",
    "rslx_ppo_update_recurrent_dc", "rslx_gae_noalloc", "rslx_linear_attention_workspace_bytes", "rslx_linear_attention",
    "rslx_linear_attention_backward_workspace_bytes", "rslx_linear_attention_backward", "rslx_linear_attention_step",
    "rslx_layer_norm", "rslx_layer_norm_backward_workspace_bytes", "rslx_layer_norm_backward",
    "rslx_gated_recurrence_workspace_bytes", "rslx_gated_recurrence", "rslx_gated_recurrence_backward_workspace_bytes",
    "rslx_gated_recurrence_backward", "rslx_gated_recurrence_step", "rslx_rms_norm", "rslx_rms_norm_e4m3",
    "rslx_rms_norm_backward_workspace_bytes", "rslx_rms_norm_backward", "rslx_muon_step_workspace_bytes",
    "rslx_muon_step",
]
GAE_NOALLOC_MAX_ENVS = 1 << 20
ATTN_MAX_DIM = 128
NORM_MAX_COLS = 16384

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librslx.so")


class RslxError(RuntimeError):
    pass


if not os.path.exists(_LIB_PATH):
    raise ImportError("librslx.so is missing at %s: build it with `python paper_2509_10771_amd/build.py`; "
                      "there is no fallback path" % _LIB_PATH)
lib = C.CDLL(_LIB_PATH)

_fp = C.POINTER(C.c_float)
_vp = C.c_void_p


class _CMlp(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("dims", C.c_int32 * (MAX_LAYERS + 1)), ("elu_alpha", C.c_float),
                ("has_log_std", C.c_int32), ("params", _vp), ("grads", _vp), ("adam_m", _vp), ("adam_v", _vp)]


class _CMemory(C.Structure):
    _fields_ = [("cell", C.c_int32), ("in_dim", C.c_int32), ("hidden", C.c_int32), ("params", _vp), ("grads", _vp),
                ("adam_m", _vp), ("adam_v", _vp)]


class _CRollout(C.Structure):
    _fields_ = [("T", C.c_int32), ("N", C.c_int32), ("Da", C.c_int32), ("Dc", C.c_int32), ("A", C.c_int32),
                ("obs_actor", _vp), ("obs_critic", _vp), ("actions", _vp), ("logp", _vp), ("values", _vp),
                ("mu", _vp), ("sigma", _vp), ("advantages", _vp), ("returns", _vp)]


class _CPpoCfg(C.Structure):
    _fields_ = [("clip", C.c_float), ("value_coef", C.c_float), ("entropy_coef", C.c_float), ("max_grad_norm", C.c_float),
                ("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("adam_eps", C.c_float),
                ("epochs", C.c_int32), ("minibatches", C.c_int32), ("use_clipped_value_loss", C.c_int32),
                ("seed", C.c_uint64), ("call_index", C.c_uint64), ("epoch_offset", C.c_int32)]


class _CSym(C.Structure):
    _fields_ = [("perm_obs_a_host", _vp), ("sign_obs_a_host", _vp), ("perm_obs_c_host", _vp), ("sign_obs_c_host", _vp),
                ("perm_act_host", _vp), ("sign_act_host", _vp),
                ("perm_obs_a", _vp), ("sign_obs_a", _vp), ("perm_obs_c", _vp), ("sign_obs_c", _vp),
                ("perm_act", _vp), ("sign_act", _vp), ("mirror_loss_coef", C.c_float)]


class _CRndTrain(C.Structure):
    _fields_ = [("target", C.POINTER(_CMlp)), ("predictor", C.POINTER(_CMlp)), ("subset_idx", _vp),
                ("n_subset", C.c_int32), ("lr", C.c_float), ("adam_step", C.POINTER(C.c_int64))]


class _CBcCfg(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("adam_eps", C.c_float),
                ("max_grad_norm", C.c_float), ("epochs", C.c_int32), ("minibatches", C.c_int32),
                ("seed", C.c_uint64), ("call_index", C.c_uint64), ("epoch_offset", C.c_int32)]


class _CTraceRecord(C.Structure):
    _fields_ = [("kernel", C.c_char * 48), ("flops", C.c_double), ("bytes", C.c_double), ("ms", C.c_float)]


class _CSeqView(C.Structure):
    _fields_ = [("data", _vp), ("step", C.c_int64), ("seq", C.c_int64), ("head", C.c_int64)]


class _CGatedRec(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("T", C.c_int32), ("N", C.c_int32), ("D", C.c_int32), ("dones", _vp), ("lengths", _vp)]


class _CMuonMatrix(C.Structure):
    _fields_ = [("w_in", _vp), ("w_out", _vp), ("grad", _vp), ("m_in", _vp), ("m_out", _vp), ("rows", C.c_int32), ("cols", C.c_int32),
                ("scale", C.c_float)]


class _CMuonCfg(C.Structure):
    _fields_ = [("lr", C.c_float), ("momentum", C.c_float), ("weight_decay", C.c_float), ("nesterov", C.c_int32), ("steps", C.c_int32)]


class _CLinearAttn(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("T", C.c_int32), ("N", C.c_int32), ("H", C.c_int32), ("Dk", C.c_int32), ("Dv", C.c_int32),
                ("scale", C.c_float), ("log_decay", _vp), ("dones", _vp), ("lengths", _vp)]


def _sig(name, restype, argtypes):
    f = getattr(lib, name)
    f.restype = restype
    f.argtypes = argtypes
    return f


_P = C.POINTER
_sig("rslx_version", C.c_int32, [])
_sig("rslx_last_error", C.c_char_p, [])
_sig("rslx_device_check", C.c_int32, [])
_sig("rslx_permutation_workspace_bytes", C.c_size_t, [C.c_int32])
_sig("rslx_permutation", C.c_int32, [C.c_uint64, C.c_uint64, C.c_int32, C.c_int32, _vp, _vp, C.c_size_t, _vp])
_sig("rslx_act_workspace_bytes", C.c_size_t, [_P(_CMlp), _P(_CMlp), C.c_int32])
_sig("rslx_act", C.c_int32, [_P(_CMlp), _P(_CMlp), _vp, _vp, C.c_int32, C.c_uint64, C.c_uint64, _vp, _vp, _vp, _vp, _vp,
                             _vp, C.c_uint32, _vp, C.c_size_t, _vp])
_sig("rslx_act_dc", C.c_int32, [_P(_CMlp), _P(_CMlp), _vp, _vp, C.c_int32, C.c_uint64, _vp, _vp, _vp, _vp, _vp, _vp,
                                _vp, C.c_uint32, _vp, C.c_size_t, _vp])
_sig("rslx_gae_workspace_bytes", C.c_size_t, [C.c_int32, C.c_int32])
_sig("rslx_gae", C.c_int32, [_vp, _vp, _vp, _vp, _vp, C.c_int32, C.c_int32, C.c_float, C.c_float, C.c_int32, _vp, _vp,
                             _vp, C.c_size_t, _vp])
_sig("rslx_gae_noalloc", C.c_int32, [_vp, _vp, _vp, _vp, _vp, C.c_int32, C.c_int32, C.c_float, C.c_float, C.c_int32, _vp, _vp, _vp])
_sig("rslx_adam_workspace_bytes", C.c_size_t, [C.c_int64])
_sig("rslx_adam_step", C.c_int32, [_vp, _vp, _vp, _vp, C.c_int64, C.c_float, C.c_float, C.c_float, C.c_float, C.c_float,
                                   _P(C.c_int64), _vp, _vp, C.c_size_t, _vp])
_sig("rslx_ppo_update_workspace_bytes", C.c_size_t, [_P(_CMlp), _P(_CMlp), _P(_CRollout), _P(_CPpoCfg), _P(_CSym), _P(_CRndTrain)])
_sig("rslx_ppo_update", C.c_int32, [_P(_CMlp), _P(_CMlp), _P(_CRollout), _P(_CPpoCfg), _P(_CSym), _P(_CRndTrain),
                                    _P(C.c_int64), _vp, _vp, C.c_size_t, _vp])
_sig("rslx_ppo_update_dc", C.c_int32, [_P(_CMlp), _P(_CMlp), _P(_CRollout), _P(_CPpoCfg), _P(_CSym), _P(_CRndTrain),
                                       _vp, _vp, _vp, C.c_size_t, _vp])
_sig("rslx_bc_update_workspace_bytes", C.c_size_t, [_P(_CMlp), _P(_CMlp), C.c_int32, _P(_CBcCfg)])
_sig("rslx_bc_update", C.c_int32, [_P(_CMlp), _P(_CMlp), _vp, _vp, _vp, C.c_int32, _P(_CBcCfg), _P(C.c_int64), _vp, _vp,
                                   C.c_size_t, _vp])
_sig("rslx_bc_update_dc", C.c_int32, [_P(_CMlp), _P(_CMlp), _vp, _vp, _vp, C.c_int32, _P(_CBcCfg), _vp, _vp, _vp,
                                      C.c_size_t, _vp])
_sig("rslx_bc_collect_workspace_bytes", C.c_size_t, [_P(_CMlp), _P(_CMlp), C.c_int32])
_sig("rslx_bc_collect", C.c_int32, [_P(_CMlp), _P(_CMlp), _vp, _vp, C.c_int32, _vp, _vp, _vp, C.c_size_t, _vp])
_sig("rslx_act_recurrent_workspace_bytes", C.c_size_t, [_P(_CMemory), _P(_CMlp), _P(_CMemory), _P(_CMlp), C.c_int32])
_sig("rslx_act_recurrent", C.c_int32, [_P(_CMemory), _P(_CMlp), _P(_CMemory), _P(_CMlp), _vp, _vp, C.c_int32, _vp, _vp, _vp, _vp,
                                       _vp, C.c_uint64, C.c_uint64, _vp, _vp, _vp, _vp, _vp, _vp, C.c_uint32, _vp,
                                       C.c_size_t, _vp])
_sig("rslx_act_recurrent_dc", C.c_int32, [_P(_CMemory), _P(_CMlp), _P(_CMemory), _P(_CMlp), _vp, _vp, C.c_int32, _vp, _vp, _vp,
                                          _vp, _vp, C.c_uint64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, C.c_uint32, _vp,
                                          C.c_size_t, _vp])
_sig("rslx_ppo_update_recurrent_dc", C.c_int32, [_P(_CMemory), _P(_CMlp), _P(_CMemory), _P(_CMlp), _P(_CRollout), _vp, _vp, _vp,
                                                 _P(_CPpoCfg), _vp, _vp, _vp, C.c_size_t, _vp])
_sig("rslx_ppo_update_recurrent_workspace_bytes", C.c_size_t, [_P(_CMemory), _P(_CMlp), _P(_CMemory), _P(_CMlp), _P(_CRollout),
                                                               _P(_CPpoCfg)])
_sig("rslx_ppo_update_recurrent", C.c_int32, [_P(_CMemory), _P(_CMlp), _P(_CMemory), _P(_CMlp), _P(_CRollout), _vp, _vp, _vp,
                                              _P(_CPpoCfg), _P(C.c_int64), _vp, _vp, C.c_size_t, _vp])
_sig("rslx_memory_step_workspace_bytes", C.c_size_t, [_P(_CMemory), C.c_int32])
_sig("rslx_memory_step", C.c_int32, [_P(_CMemory), _vp, C.c_int32, _vp, _vp, _vp, _vp, _vp, C.c_size_t, _vp])
_sig("rslx_bc_update_recurrent_workspace_bytes", C.c_size_t, [_P(_CMemory), _P(_CMlp), C.c_int32, C.c_int32, _P(_CBcCfg)])
_sig("rslx_bc_update_recurrent", C.c_int32, [_P(_CMemory), _P(_CMlp), _vp, _vp, _vp, _vp, C.c_int32, C.c_int32, _P(_CBcCfg),
                                             _P(C.c_int64), _vp, _vp, C.c_size_t, _vp])
_sig("rslx_sym_augment", C.c_int32, [_P(_CSym), _vp, _vp, C.c_int32, C.c_int32, C.c_int32, _vp, _vp, _vp])
_sig("rslx_rnd_workspace_bytes", C.c_size_t, [_P(_CMlp), C.c_int32])
_sig("rslx_rnd", C.c_int32, [_P(_CMlp), _P(_CMlp), _vp, C.c_int32, C.c_int32, _vp, C.c_int32, _vp, C.c_float, C.c_int32,
                             _vp, _vp, _vp, C.c_size_t, _vp])


_sig("rslx_linear_attention_workspace_bytes", C.c_size_t, [_P(_CLinearAttn)])
_sig("rslx_linear_attention", C.c_int32, [_P(_CLinearAttn), _P(_CSeqView), _P(_CSeqView), _P(_CSeqView), _vp, _P(_CSeqView), _vp, _vp,
                                          C.c_size_t, _vp])
_sig("rslx_linear_attention_backward_workspace_bytes", C.c_size_t, [_P(_CLinearAttn)])
_sig("rslx_linear_attention_backward", C.c_int32, [_P(_CLinearAttn), _P(_CSeqView), _P(_CSeqView), _P(_CSeqView), _vp, _P(_CSeqView), _vp,
                                                   _P(_CSeqView), _P(_CSeqView), _P(_CSeqView), _vp, _vp, C.c_size_t, _vp])
_sig("rslx_linear_attention_step", C.c_int32, [_P(_CLinearAttn), _P(_CSeqView), _P(_CSeqView), _P(_CSeqView), _vp, _vp, _vp, _P(_CSeqView),
                                               _vp])
_sig("rslx_layer_norm", C.c_int32, [C.c_int32, _vp, C.c_int64, C.c_int64, C.c_int32, _vp, _vp, C.c_float, _vp, C.c_int64, _vp, _vp, _vp])
_sig("rslx_layer_norm_backward_workspace_bytes", C.c_size_t, [C.c_int64, C.c_int32])
_sig("rslx_layer_norm_backward", C.c_int32, [C.c_int32, _vp, C.c_int64, _vp, C.c_int64, C.c_int64, C.c_int32, _vp, _vp, _vp, _vp, C.c_int64, _vp,
                                             _vp, _vp, C.c_size_t, _vp])
_sig("rslx_gated_recurrence_workspace_bytes", C.c_size_t, [_P(_CGatedRec)])
_sig("rslx_gated_recurrence", C.c_int32, [_P(_CGatedRec), _P(_CSeqView), _P(_CSeqView), _vp, _P(_CSeqView), _vp, _vp, C.c_size_t, _vp])
_sig("rslx_gated_recurrence_backward_workspace_bytes", C.c_size_t, [_P(_CGatedRec)])
_sig("rslx_gated_recurrence_backward", C.c_int32, [_P(_CGatedRec), _P(_CSeqView), _P(_CSeqView), _vp, _P(_CSeqView), _vp, _P(_CSeqView),
                                                   _P(_CSeqView), _vp, _vp, C.c_size_t, _vp])
_sig("rslx_gated_recurrence_step", C.c_int32, [_P(_CGatedRec), _P(_CSeqView), _P(_CSeqView), _vp, _vp, _vp, _P(_CSeqView), _vp])
_sig("rslx_rms_norm", C.c_int32, [C.c_int32, _vp, C.c_int64, _vp, C.c_int64, C.c_int64, C.c_int32, _vp, C.c_float, _vp, C.c_int64, _vp, C.c_int64,
                                  _vp, _vp])
_sig("rslx_rms_norm_e4m3", C.c_int32, [C.c_int32, _vp, C.c_int64, _vp, C.c_int64, C.c_int64, C.c_int32, _vp, C.c_float, _vp, C.c_int64, _vp,
                                       C.c_int64, _vp, _vp, _vp])
_sig("rslx_rms_norm_backward_workspace_bytes", C.c_size_t, [C.c_int64, C.c_int32])
_sig("rslx_rms_norm_backward", C.c_int32, [C.c_int32, _vp, C.c_int64, _vp, C.c_int64, C.c_int64, C.c_int32, _vp, _vp, _vp, C.c_int64, _vp, C.c_int64,
                                           _vp, _vp, C.c_size_t, _vp])
_sig("rslx_muon_step_workspace_bytes", C.c_size_t, [_P(_CMuonMatrix), C.c_int32, _P(_CMuonCfg)])
_sig("rslx_muon_step", C.c_int32, [_P(_CMuonMatrix), C.c_int32, _P(_CMuonCfg), _vp, C.c_size_t, _vp])
_sig("rslx_trace_begin", C.c_int32, [C.c_int32])
_sig("rslx_trace_end", C.c_int32, [_P(_CTraceRecord), C.c_int32, _P(C.c_int32)])


def _check(rc, what):
    if rc != 0:
        raise RslxError("%s failed with status %d: %s" % (what, rc, lib.rslx_last_error().decode()))


def _ptr(t):
    """Device (or host) address of a contiguous tensor; None -> NULL."""
    if t is None:
        return None
    assert t.is_contiguous(), "rslx needs contiguous tensors"
    return t.data_ptr()


def _stream():
    """torch's current stream; without a GPU (host-side argument checks only) the NULL stream.  Once torch runs on the GPU its
    handle is asked for directly: 0.3 us a call, where is_available() and a Stream object take 4.6 of a small call's 11."""
    if torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None


def workspace(nbytes, device="cuda"):
    """Device scratch buffer for the *_workspace_bytes() queries."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


class Mlp:
    """A network over flat device tensors (layout in include/rslx.h)."""

    def __init__(self, dims, params, trainable=False, has_log_std=False, elu_alpha=1.0):
        self.dims = tuple(int(d) for d in dims)
        self.has_log_std = bool(has_log_std)
        n = sum(i * o + o for i, o in zip(self.dims[:-1], self.dims[1:])) + (self.dims[-1] if has_log_std else 0)
        assert params.dtype == torch.float32 and params.numel() == n, (params.numel(), n)
        self.params = params
        self.grads = torch.zeros_like(params) if trainable else None
        self.adam_m = torch.zeros_like(params) if trainable else None
        self.adam_v = torch.zeros_like(params) if trainable else None
        self.elu_alpha = float(elu_alpha)

    @property
    def c(self):
        s = _CMlp()
        s.n_layers = len(self.dims) - 1
        for i, d in enumerate(self.dims):
            s.dims[i] = d
        s.elu_alpha = self.elu_alpha
        s.has_log_std = int(self.has_log_std)
        s.params = _ptr(self.params)
        s.grads = _ptr(self.grads)
        s.adam_m = _ptr(self.adam_m)
        s.adam_v = _ptr(self.adam_v)
        return s


CELL_GRU, CELL_LSTM = 0, 1


class Memory:
    """Recurrent memory over a flat device buffer: W_ih [in, G H], b_ih [G H], W_hh [H, G H], b_hh [G H]
    (GRU: G = 3, state width H; LSTM: G = 4, packed state [h | c] of width 2 H)."""

    def __init__(self, cell, in_dim, hidden, params, trainable=False):
        self.cell, self.in_dim, self.hidden = int(cell), int(in_dim), int(hidden)
        self.gates = 4 if self.cell == CELL_LSTM else 3
        self.state_width = 2 * self.hidden if self.cell == CELL_LSTM else self.hidden
        assert params.numel() == self.gates * self.hidden * (self.in_dim + self.hidden + 2)
        self.params = params
        self.grads = torch.zeros_like(params) if trainable else None
        self.adam_m = torch.zeros_like(params) if trainable else None
        self.adam_v = torch.zeros_like(params) if trainable else None

    @property
    def c(self):
        return _CMemory(self.cell, self.in_dim, self.hidden, _ptr(self.params), _ptr(self.grads), _ptr(self.adam_m),
                        _ptr(self.adam_v))


def Gru(in_dim, hidden, params, trainable=False):
    return Memory(CELL_GRU, in_dim, hidden, params, trainable)


def Lstm(in_dim, hidden, params, trainable=False):
    return Memory(CELL_LSTM, in_dim, hidden, params, trainable)


class Rollout:
    def __init__(self, T, N, obs_actor, obs_critic, actions, logp, values, mu, sigma, advantages, returns):
        self.T, self.N = int(T), int(N)
        self.t = dict(obs_actor=obs_actor, obs_critic=obs_critic, actions=actions, logp=logp, values=values, mu=mu,
                      sigma=sigma, advantages=advantages, returns=returns)
        B = self.T * self.N
        self.Da, self.Dc, self.A = obs_actor.numel() // B, obs_critic.numel() // B, actions.numel() // B

    @property
    def c(self):
        s = _CRollout(self.T, self.N, self.Da, self.Dc, self.A)
        for k, v in self.t.items():
            setattr(s, k, _ptr(v))
        return s


class PpoCfg:
    def __init__(self, clip=0.2, value_coef=1.0, entropy_coef=0.01, max_grad_norm=1.0, lr=1e-3, beta1=0.9, beta2=0.999,
                 adam_eps=1e-8, epochs=5, minibatches=4, use_clipped_value_loss=True, seed=0, call_index=0, epoch_offset=0):
        self.c = _CPpoCfg(clip, value_coef, entropy_coef, max_grad_norm, lr, beta1, beta2, adam_eps, epochs, minibatches,
                          int(use_clipped_value_loss), seed, call_index, epoch_offset)


class BcCfg:
    def __init__(self, lr=1e-3, beta1=0.9, beta2=0.999, adam_eps=1e-8, max_grad_norm=0.0, epochs=2, minibatches=4, seed=0,
                 call_index=0, epoch_offset=0):
        self.c = _CBcCfg(lr, beta1, beta2, adam_eps, max_grad_norm, epochs, minibatches, seed, call_index, epoch_offset)


class Sym:
    """Mirror maps: host copies (int32 / float32 CPU tensors) plus device copies (device=None: none; rslx_ppo_update
    then uploads the host copies itself)."""

    def __init__(self, perm_obs_a, sign_obs_a, perm_obs_c, sign_obs_c, perm_act, sign_act, mirror_loss_coef=1.0, device="cuda"):
        host = [torch.as_tensor(perm_obs_a, dtype=torch.int32).contiguous(), torch.as_tensor(sign_obs_a, dtype=torch.float32).contiguous(),
                torch.as_tensor(perm_obs_c, dtype=torch.int32).contiguous(), torch.as_tensor(sign_obs_c, dtype=torch.float32).contiguous(),
                torch.as_tensor(perm_act, dtype=torch.int32).contiguous(), torch.as_tensor(sign_act, dtype=torch.float32).contiguous()]
        self.host = host
        self.dev = [h.to(device) for h in host] if device is not None else [None] * 6
        self.mirror_loss_coef = float(mirror_loss_coef)

    @property
    def c(self):
        s = _CSym()
        names = ["perm_obs_a", "sign_obs_a", "perm_obs_c", "sign_obs_c", "perm_act", "sign_act"]
        for n, h, d in zip(names, self.host, self.dev):
            setattr(s, n + "_host", _ptr(h))
            setattr(s, n, _ptr(d))
        s.mirror_loss_coef = self.mirror_loss_coef
        return s


class RndTrain:
    def __init__(self, target, predictor, subset_idx=None, lr=1e-3, adam_step=0):
        self.target, self.predictor, self.subset_idx, self.lr = target, predictor, subset_idx, float(lr)
        self.step = C.c_int64(int(adam_step))

    def c(self):
        self._ct, self._cp = self.target.c, self.predictor.c
        s = _CRndTrain(C.pointer(self._ct), C.pointer(self._cp), _ptr(self.subset_idx),
                       self.target.dims[0], self.lr, C.pointer(self.step))
        return s


def _ref(x):
    return None if x is None else C.byref(x)


def rslx_version():
    return lib.rslx_version()


def rslx_device_check():
    _check(lib.rslx_device_check(), "rslx_device_check")


def rslx_permutation_workspace_bytes(B):
    return lib.rslx_permutation_workspace_bytes(B)


def rslx_permutation(seed, call_index, epoch, B, perm_out, ws):
    _check(lib.rslx_permutation(seed, call_index, epoch, B, _ptr(perm_out), _ptr(ws), ws.numel(), _stream()), "rslx_permutation")


def rslx_act_workspace_bytes(actor, critic, N):
    return lib.rslx_act_workspace_bytes(_ref(actor.c) if actor is not None else None, _ref(critic.c), N)


def rslx_act(actor, critic, obs_actor, obs_critic, N, seed, step, eps, actions, logp, values, mu, sigma, flags, ws):
    ca = actor.c if actor is not None else None
    cc = critic.c
    _check(lib.rslx_act(_ref(ca), _ref(cc), _ptr(obs_actor), _ptr(obs_critic), N, seed, step, _ptr(eps), _ptr(actions),
                        _ptr(logp), _ptr(values), _ptr(mu), _ptr(sigma), flags, _ptr(ws), ws.numel(), _stream()), "rslx_act")


def dev_counters(act_step=0, call_index=0, adam_step=0, rnd_adam_step=0, device="cuda"):
    """rslx_dev_counters in device memory: int64 tensor [act_step, call_index, adam_step, rnd_adam_step]."""
    return torch.tensor([act_step, call_index, adam_step, rnd_adam_step], dtype=torch.int64, device=device)


def rslx_act_dc(actor, critic, obs_actor, obs_critic, N, seed, counters, eps, actions, logp, values, mu, sigma, flags, ws):
    """counters: int64 device tensor of 4 (dev_counters())."""
    ca = actor.c if actor is not None else None
    cc = critic.c
    _check(lib.rslx_act_dc(_ref(ca), _ref(cc), _ptr(obs_actor), _ptr(obs_critic), N, seed, _ptr(counters), _ptr(eps),
                           _ptr(actions), _ptr(logp), _ptr(values), _ptr(mu), _ptr(sigma), flags, _ptr(ws), ws.numel(),
                           _stream()), "rslx_act_dc")


def rslx_gae_workspace_bytes(T, N):
    return lib.rslx_gae_workspace_bytes(T, N)


def rslx_gae(rewards, values, last_values, dones, timeouts, T, N, gamma, lam, normalize_adv, advantages, returns, ws):
    _check(lib.rslx_gae(_ptr(rewards), _ptr(values), _ptr(last_values), _ptr(dones), _ptr(timeouts), T, N, gamma, lam,
                        int(normalize_adv), _ptr(advantages), _ptr(returns), _ptr(ws), ws.numel() if ws is not None else 0,
                        _stream()), "rslx_gae")


def rslx_gae_noalloc(rewards, values, last_values, dones, timeouts, T, N, gamma, lam, normalize_adv, advantages, returns):
    _check(lib.rslx_gae_noalloc(_ptr(rewards), _ptr(values), _ptr(last_values), _ptr(dones), _ptr(timeouts), T, N, gamma, lam,
                                int(normalize_adv), _ptr(advantages), _ptr(returns), _stream()), "rslx_gae_noalloc")


def rslx_adam_workspace_bytes(n):
    return lib.rslx_adam_workspace_bytes(n)


def rslx_adam_step(params, grads, m, v, n, lr, beta1, beta2, eps, max_grad_norm, adam_step, grad_norm_out, ws):
    """adam_step: ctypes.c_int64, updated in place."""
    _check(lib.rslx_adam_step(_ptr(params), _ptr(grads), _ptr(m), _ptr(v), n, lr, beta1, beta2, eps, max_grad_norm,
                              C.byref(adam_step), _ptr(grad_norm_out), _ptr(ws), ws.numel(), _stream()), "rslx_adam_step")


def rslx_ppo_update_workspace_bytes(actor, critic, rollout, cfg, sym=None, rnd=None):
    ca, cc, cr = actor.c, critic.c, rollout.c
    cs = sym.c if sym is not None else None
    cn = rnd.c() if rnd is not None else None
    n = lib.rslx_ppo_update_workspace_bytes(_ref(ca), _ref(cc), _ref(cr), _ref(cfg.c), _ref(cs), _ref(cn))
    if n == 0:
        raise RslxError("rslx_ppo_update_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_ppo_update(actor, critic, rollout, cfg, sym, rnd, adam_step, stats, ws):
    """adam_step: ctypes.c_int64, updated in place."""
    ca, cc, cr = actor.c, critic.c, rollout.c
    cs = sym.c if sym is not None else None
    cn = rnd.c() if rnd is not None else None
    _check(lib.rslx_ppo_update(_ref(ca), _ref(cc), _ref(cr), _ref(cfg.c), _ref(cs), _ref(cn), C.byref(adam_step),
                               _ptr(stats), _ptr(ws), ws.numel() if ws is not None else 0, _stream()), "rslx_ppo_update")


def rslx_ppo_update_dc(actor, critic, rollout, cfg, sym, rnd, counters, stats, ws):
    """counters: int64 device tensor of 4 (dev_counters()), advanced by the call's own kernels."""
    ca, cc, cr = actor.c, critic.c, rollout.c
    cs = sym.c if sym is not None else None
    cn = rnd.c() if rnd is not None else None
    _check(lib.rslx_ppo_update_dc(_ref(ca), _ref(cc), _ref(cr), _ref(cfg.c), _ref(cs), _ref(cn), _ptr(counters),
                                  _ptr(stats), _ptr(ws), ws.numel() if ws is not None else 0, _stream()), "rslx_ppo_update_dc")


def rslx_bc_update_workspace_bytes(student, teacher, B, cfg):
    cs = student.c
    ct = teacher.c if teacher is not None else None
    n = lib.rslx_bc_update_workspace_bytes(_ref(cs), _ref(ct), B, _ref(cfg.c))
    if n == 0:
        raise RslxError("rslx_bc_update_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_bc_update(student, teacher, obs_student, obs_teacher, targets, B, cfg, adam_step, stats, ws):
    cs = student.c
    ct = teacher.c if teacher is not None else None
    _check(lib.rslx_bc_update(_ref(cs), _ref(ct), _ptr(obs_student), _ptr(obs_teacher), _ptr(targets), B, _ref(cfg.c),
                              C.byref(adam_step), _ptr(stats), _ptr(ws), ws.numel() if ws is not None else 0, _stream()),
           "rslx_bc_update")


def rslx_bc_update_dc(student, teacher, obs_student, obs_teacher, targets, B, cfg, counters, stats, ws):
    """counters: int64 device tensor of 4 (dev_counters()); call_index and adam_step are used."""
    cs = student.c
    ct = teacher.c if teacher is not None else None
    _check(lib.rslx_bc_update_dc(_ref(cs), _ref(ct), _ptr(obs_student), _ptr(obs_teacher), _ptr(targets), B, _ref(cfg.c),
                                 _ptr(counters), _ptr(stats), _ptr(ws), ws.numel() if ws is not None else 0, _stream()),
           "rslx_bc_update_dc")


def rslx_bc_collect_workspace_bytes(student, teacher, N):
    return lib.rslx_bc_collect_workspace_bytes(_ref(student.c), _ref(teacher.c), N)


def rslx_bc_collect(student, teacher, obs_student, obs_teacher, N, actions, targets, ws):
    cs = student.c if student is not None else None
    ct = teacher.c if teacher is not None else None
    _check(lib.rslx_bc_collect(_ref(cs), _ref(ct), _ptr(obs_student), _ptr(obs_teacher), N, _ptr(actions), _ptr(targets),
                               _ptr(ws), ws.numel() if ws is not None else 0, _stream()), "rslx_bc_collect")


def rslx_act_recurrent_workspace_bytes(gru_actor, actor, gru_critic, critic, N):
    ga = gru_actor.c if gru_actor is not None else None
    ca = actor.c if actor is not None else None
    return lib.rslx_act_recurrent_workspace_bytes(_ref(ga), _ref(ca), _ref(gru_critic.c), _ref(critic.c), N)


def rslx_act_recurrent(gru_actor, actor, gru_critic, critic, obs_actor, obs_critic, N, h_actor, h_critic, reset, h0_actor_out,
                       h0_critic_out, seed, step, eps, actions, logp, values, mu, sigma, flags, ws):
    ga = gru_actor.c if gru_actor is not None else None
    ca = actor.c if actor is not None else None
    _check(lib.rslx_act_recurrent(_ref(ga), _ref(ca), _ref(gru_critic.c), _ref(critic.c), _ptr(obs_actor), _ptr(obs_critic), N,
                                  _ptr(h_actor), _ptr(h_critic), _ptr(reset), _ptr(h0_actor_out), _ptr(h0_critic_out), seed,
                                  step, _ptr(eps), _ptr(actions), _ptr(logp), _ptr(values), _ptr(mu), _ptr(sigma), flags,
                                  _ptr(ws), ws.numel() if ws is not None else 0, _stream()), "rslx_act_recurrent")


def rslx_act_recurrent_dc(gru_actor, actor, gru_critic, critic, obs_actor, obs_critic, N, h_actor, h_critic, reset, h0_actor_out,
                          h0_critic_out, seed, counters, eps, actions, logp, values, mu, sigma, flags, ws):
    ga = gru_actor.c if gru_actor is not None else None
    ca = actor.c if actor is not None else None
    _check(lib.rslx_act_recurrent_dc(_ref(ga), _ref(ca), _ref(gru_critic.c), _ref(critic.c), _ptr(obs_actor), _ptr(obs_critic), N,
                                     _ptr(h_actor), _ptr(h_critic), _ptr(reset), _ptr(h0_actor_out), _ptr(h0_critic_out), seed,
                                     _ptr(counters), _ptr(eps), _ptr(actions), _ptr(logp), _ptr(values), _ptr(mu), _ptr(sigma),
                                     flags, _ptr(ws), ws.numel() if ws is not None else 0, _stream()), "rslx_act_recurrent_dc")


def rslx_ppo_update_recurrent_dc(gru_actor, actor, gru_critic, critic, rollout, dones, h0_actor, h0_critic, cfg, counters, stats, ws):
    _check(lib.rslx_ppo_update_recurrent_dc(_ref(gru_actor.c), _ref(actor.c), _ref(gru_critic.c), _ref(critic.c), _ref(rollout.c),
                                            _ptr(dones), _ptr(h0_actor), _ptr(h0_critic), _ref(cfg.c), _ptr(counters),
                                            _ptr(stats), _ptr(ws), ws.numel() if ws is not None else 0, _stream()),
           "rslx_ppo_update_recurrent_dc")


def rslx_ppo_update_recurrent_workspace_bytes(gru_actor, actor, gru_critic, critic, rollout, cfg):
    n = lib.rslx_ppo_update_recurrent_workspace_bytes(_ref(gru_actor.c), _ref(actor.c), _ref(gru_critic.c), _ref(critic.c),
                                                      _ref(rollout.c), _ref(cfg.c))
    if n == 0:
        raise RslxError("rslx_ppo_update_recurrent_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_ppo_update_recurrent(gru_actor, actor, gru_critic, critic, rollout, dones, h0_actor, h0_critic, cfg, adam_step, stats, ws):
    """adam_step: ctypes.c_int64, updated in place."""
    _check(lib.rslx_ppo_update_recurrent(_ref(gru_actor.c), _ref(actor.c), _ref(gru_critic.c), _ref(critic.c), _ref(rollout.c),
                                         _ptr(dones), _ptr(h0_actor), _ptr(h0_critic), _ref(cfg.c), C.byref(adam_step),
                                         _ptr(stats), _ptr(ws), ws.numel() if ws is not None else 0, _stream()),
           "rslx_ppo_update_recurrent")


def rslx_memory_step_workspace_bytes(mem, N):
    return lib.rslx_memory_step_workspace_bytes(_ref(mem.c), N)


def rslx_memory_step(mem, obs, N, state, reset, s0_out, h_dense_out, ws):
    _check(lib.rslx_memory_step(_ref(mem.c), _ptr(obs), N, _ptr(state), _ptr(reset), _ptr(s0_out), _ptr(h_dense_out), _ptr(ws),
                                ws.numel() if ws is not None else 0, _stream()), "rslx_memory_step")


def rslx_bc_update_recurrent_workspace_bytes(gru, student, T, N, cfg):
    n = lib.rslx_bc_update_recurrent_workspace_bytes(_ref(gru.c), _ref(student.c), T, N, _ref(cfg.c))
    if n == 0:
        raise RslxError("rslx_bc_update_recurrent_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_bc_update_recurrent(gru, student, obs_student, targets, dones, h0, T, N, cfg, adam_step, stats, ws):
    """adam_step: ctypes.c_int64, updated in place."""
    _check(lib.rslx_bc_update_recurrent(_ref(gru.c), _ref(student.c), _ptr(obs_student), _ptr(targets), _ptr(dones), _ptr(h0),
                                        T, N, _ref(cfg.c), C.byref(adam_step), _ptr(stats), _ptr(ws),
                                        ws.numel() if ws is not None else 0, _stream()), "rslx_bc_update_recurrent")


def rslx_sym_augment(sym, obs_in, act_in, B, D, A, obs_out, act_out):
    cs = sym.c
    _check(lib.rslx_sym_augment(_ref(cs), _ptr(obs_in), _ptr(act_in), B, D, A, _ptr(obs_out), _ptr(act_out), _stream()),
           "rslx_sym_augment")


def rslx_rnd_workspace_bytes(target, N):
    return lib.rslx_rnd_workspace_bytes(_ref(target.c), N)


def rslx_rnd(target, predictor, obs, N, D, subset_idx, n_subset, running, weight, update_stats, r_int_out, rewards_inout, ws):
    ct, cp = target.c, predictor.c
    _check(lib.rslx_rnd(_ref(ct), _ref(cp), _ptr(obs), N, D, _ptr(subset_idx), n_subset, _ptr(running), weight,
                        int(update_stats), _ptr(r_int_out), _ptr(rewards_inout), _ptr(ws), ws.numel(), _stream()), "rslx_rnd")


_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _int32(name, n):
    """The number itself; ctypes would cut what has more than 32 bits off without a word."""
    if not -1 << 31 <= n < 1 << 31:
        raise RslxError("%s = %d has more than 32 bits" % (name, n))
    return int(n)


class LinearAttn:
    """Sizes and constants of a linear-attention layer (struct rslx_linear_attn): T steps of N sequences, H heads, keys Dk and values
    Dv wide, in `dtype`; log_decay [H] float32; dones uint8 [T, N] and lengths int32 [N] or None."""

    def __init__(self, dtype, T, N, H, Dk, Dv, log_decay, scale=1.0, dones=None, lengths=None):
        if dtype not in _DTYPES:
            raise RslxError("LinearAttn: dtype %s is not one of float32, bfloat16, float16" % dtype)
        for name, t, want, n in (("log_decay", log_decay, torch.float32, H), ("dones", dones, torch.uint8, T * N), ("lengths", lengths, torch.int32, N)):
            if t is not None and (t.dtype != want or t.numel() != n):
                raise RslxError("LinearAttn: %s has %d values of %s, %d of %s are needed" % (name, t.numel(), t.dtype, n, want))
        self.dtype = dtype
        self.T, self.N, self.H, self.Dk, self.Dv = (_int32(name, n) for name, n in (("T", T), ("N", N), ("H", H), ("Dk", Dk), ("Dv", Dv)))
        self.scale, self.log_decay, self.dones, self.lengths = float(scale), log_decay, dones, lengths
        self._shapes, self._state = {w: (self.T, self.N, self.H, w) for w in (self.Dk, self.Dv)}, self.N * self.H * self.Dk * self.Dv
        self.c = _CLinearAttn(_DTYPES[dtype], self.T, self.N, self.H, self.Dk, self.Dv, self.scale, _ptr(log_decay), _ptr(dones), _ptr(lengths))

    def view(self, name, t, width):
        """t [T, N, H, width] of any strides with its values side by side -> struct rslx_seq_view."""
        if t.dtype is not self.dtype or t.shape != self._shapes[width]:
            raise RslxError("%s is %s %s, %s %s is needed" % (name, t.dtype, tuple(t.shape), self.dtype, (self.T, self.N, self.H, width)))
        step, seq, head, one = t.stride()
        if one != 1 and width > 1 and t.numel() > 0:
            raise RslxError("%s: the values of a row must lie side by side" % name)
        return _CSeqView(t.data_ptr(), step, seq, head)

    def state(self, name, t):
        """t [N, H, Dk, Dv] float32, contiguous, or None -> address."""
        if t is None:
            return None
        if t.dtype is not torch.float32 or t.numel() != self._state:
            raise RslxError("%s has %d values of %s, %d of float32 are needed" % (name, t.numel(), t.dtype, self._state))
        assert t.is_contiguous(), "rslx needs contiguous tensors"
        return t.data_ptr()


def rslx_linear_attention_workspace_bytes(la):
    n = lib.rslx_linear_attention_workspace_bytes(C.byref(la.c))
    if n == 0:
        raise RslxError("rslx_linear_attention_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_linear_attention(la, q, k, v, s0, o, s_last, ws):
    """q, k [T, N, H, Dk], v, o [T, N, H, Dv]; s0, s_last [N, H, Dk, Dv] float32 or None."""
    _check(lib.rslx_linear_attention(la.c, la.view("q", q, la.Dk), la.view("k", k, la.Dk), la.view("v", v, la.Dv), la.state("s0", s0),
                                     la.view("o", o, la.Dv), la.state("s_last", s_last), _ptr(ws), ws.numel() if ws is not None else 0,
                                     _stream()), "rslx_linear_attention")


def rslx_linear_attention_backward_workspace_bytes(la):
    n = lib.rslx_linear_attention_backward_workspace_bytes(C.byref(la.c))
    if n == 0:
        raise RslxError("rslx_linear_attention_backward_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_linear_attention_backward(la, q, k, v, s0, do, ds_last, dq, dk, dv, ds0, ws):
    """Gradients of rslx_linear_attention from do [T, N, H, Dv] and ds_last [N, H, Dk, Dv] (or None)."""
    _check(lib.rslx_linear_attention_backward(la.c, la.view("q", q, la.Dk), la.view("k", k, la.Dk), la.view("v", v, la.Dv),
                                              la.state("s0", s0), la.view("do", do, la.Dv), la.state("ds_last", ds_last),
                                              la.view("dq", dq, la.Dk), la.view("dk", dk, la.Dk), la.view("dv", dv, la.Dv),
                                              la.state("ds0", ds0), _ptr(ws), ws.numel() if ws is not None else 0, _stream()),
           "rslx_linear_attention_backward")


def rslx_linear_attention_step(la, q, k, v, reset, s_in, s_out, o):
    """One step (la.T == 1): q, k [1, N, H, Dk], v, o [1, N, H, Dv]; reset uint8 of N values or None; s_in (or None), s_out [N, H, Dk, Dv]."""
    if reset is not None and (reset.dtype != torch.uint8 or reset.numel() != la.N):
        raise RslxError("reset has %d values of %s, %d of uint8 are needed" % (reset.numel(), reset.dtype, la.N))
    _check(lib.rslx_linear_attention_step(la.c, la.view("q", q, la.Dk), la.view("k", k, la.Dk), la.view("v", v, la.Dv), _ptr(reset),
                                          la.state("s_in", s_in), la.state("s_out", s_out), la.view("o", o, la.Dv), _stream()),
           "rslx_linear_attention_step")


def _matrix(name, t):
    """A matrix [rows, cols] -> (type's code, its type, its shape)."""
    code, shape = _DTYPES.get(t.dtype), t.shape
    if code is None or len(shape) != 2:
        raise RslxError("%s is %s %s, a matrix of float32, bfloat16 or float16 is needed" % (name, t.dtype, tuple(shape)))
    if shape[1] > NORM_MAX_COLS:                               # (the C call's number of columns has 32 bits)
        raise RslxError("%s has %d columns, 1 to %d columns are taken" % (name, shape[1], NORM_MAX_COLS))
    return code, t.dtype, shape


def _rows(name, t, dtype, shape):
    """A matrix of that type and shape, or None, whose rows may lie apart -> (address, distance)."""
    if t is None:
        return None, 0
    if t.dtype is not dtype or t.shape != shape:
        raise RslxError("%s is %s %s, %s %s is needed" % (name, t.dtype, tuple(t.shape), dtype, tuple(shape)))
    ld, one = t.stride()
    if one != 1 and shape[1] > 1 and shape[0] > 0:
        raise RslxError("%s: the values of a row must lie side by side" % name)
    return t.data_ptr(), ld


def _f32(name, t, n):
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != n:
        raise RslxError("%s has %d values of %s, %d of float32 are needed" % (name, t.numel(), t.dtype, n))
    assert t.is_contiguous(), "rslx needs contiguous tensors"
    return t.data_ptr()


def rslx_layer_norm(x, weight, bias, eps, y, mean, rstd):
    """x, y [rows, cols]; weight, bias [cols] and mean, rstd [rows] float32 or None."""
    code, dtype, shape = _matrix("x", x)
    rows, cols = shape
    (px, ldx), (py, ldy) = _rows("x", x, dtype, shape), _rows("y", y, dtype, shape)
    _check(lib.rslx_layer_norm(code, px, ldx, rows, cols, _f32("weight", weight, cols), _f32("bias", bias, cols), eps, py, ldy,
                               _f32("mean", mean, rows), _f32("rstd", rstd, rows), _stream()), "rslx_layer_norm")


def rslx_layer_norm_backward_workspace_bytes(rows, cols):
    n = lib.rslx_layer_norm_backward_workspace_bytes(rows, _int32("cols", cols))
    if n == 0:
        raise RslxError("rslx_layer_norm_backward_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, ws):
    """dy, x, dx [rows, cols]; mean, rstd [rows] as rslx_layer_norm leaves them; dx, dweight, dbias or None."""
    code, dtype, shape = _matrix("x", x)
    rows, cols = shape
    (px, ldx), (pd, lddy), (pg, lddx) = _rows("x", x, dtype, shape), _rows("dy", dy, dtype, shape), _rows("dx", dx, dtype, shape)
    _check(lib.rslx_layer_norm_backward(code, pd, lddy, px, ldx, rows, cols, _f32("weight", weight, cols), _f32("mean", mean, rows),
                                        _f32("rstd", rstd, rows), pg, lddx, _f32("dweight", dweight, cols), _f32("dbias", dbias, cols), _ptr(ws),
                                        ws.numel() if ws is not None else 0, _stream()), "rslx_layer_norm_backward")


class GatedRec:
    """Sizes of a gated linear recurrence (struct rslx_gated_rec): T steps of N sequences, D channels, in `dtype`; dones uint8 [T, N] and
    lengths int32 [N] or None."""

    def __init__(self, dtype, T, N, D, dones=None, lengths=None):
        if dtype not in _DTYPES:
            raise RslxError("GatedRec: dtype %s is not one of float32, bfloat16, float16" % dtype)
        for name, t, want, n in (("dones", dones, torch.uint8, T * N), ("lengths", lengths, torch.int32, N)):
            if t is not None and (t.dtype != want or t.numel() != n):
                raise RslxError("GatedRec: %s has %d values of %s, %d of %s are needed" % (name, t.numel(), t.dtype, n, want))
        self.dtype, self.dones, self.lengths = dtype, dones, lengths
        self.T, self.N, self.D = (_int32(name, n) for name, n in (("T", T), ("N", N), ("D", D)))
        self._shape = (self.T, self.N, self.D)
        self.c = _CGatedRec(_DTYPES[dtype], self.T, self.N, self.D, _ptr(dones), _ptr(lengths))

    def view(self, name, t):
        """t [T, N, D] of any strides with its values side by side -> struct rslx_seq_view."""
        if t.dtype is not self.dtype or t.shape != self._shape:
            raise RslxError("%s is %s %s, %s %s is needed" % (name, t.dtype, tuple(t.shape), self.dtype, self._shape))
        step, seq, one = t.stride()
        if one != 1 and self.D > 1 and t.numel() > 0:
            raise RslxError("%s: the values of a row must lie side by side" % name)
        return _CSeqView(t.data_ptr(), step, seq, 0)

    def state(self, name, t):
        """t [N, D] float32, contiguous, or None -> address."""
        return _f32(name, t, self.N * self.D)


def rslx_gated_recurrence_workspace_bytes(gr):
    n = lib.rslx_gated_recurrence_workspace_bytes(C.byref(gr.c))
    if n == 0:
        raise RslxError("rslx_gated_recurrence_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_gated_recurrence(gr, x, g, s0, h, s_last, ws):
    """x, g, h [T, N, D]; s0, s_last [N, D] float32 or None."""
    _check(lib.rslx_gated_recurrence(gr.c, gr.view("x", x), gr.view("g", g), gr.state("s0", s0), gr.view("h", h), gr.state("s_last", s_last), _ptr(ws),
                                     ws.numel() if ws is not None else 0, _stream()), "rslx_gated_recurrence")


def rslx_gated_recurrence_backward_workspace_bytes(gr):
    n = lib.rslx_gated_recurrence_backward_workspace_bytes(C.byref(gr.c))
    if n == 0:
        raise RslxError("rslx_gated_recurrence_backward_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_gated_recurrence_backward(gr, x, g, s0, dh, ds_last, dx, dg, ds0, ws):
    """Gradients of rslx_gated_recurrence from dh [T, N, D] and ds_last [N, D] (or None)."""
    _check(lib.rslx_gated_recurrence_backward(gr.c, gr.view("x", x), gr.view("g", g), gr.state("s0", s0), gr.view("dh", dh), gr.state("ds_last", ds_last),
                                              gr.view("dx", dx), gr.view("dg", dg), gr.state("ds0", ds0), _ptr(ws),
                                              ws.numel() if ws is not None else 0, _stream()), "rslx_gated_recurrence_backward")


def rslx_gated_recurrence_step(gr, x, g, reset, s_in, s_out, h):
    """One step (gr.T == 1): x, g, h [1, N, D]; reset uint8 of N values or None; s_in (or None), s_out [N, D]."""
    if reset is not None and (reset.dtype != torch.uint8 or reset.numel() != gr.N):
        raise RslxError("reset has %d values of %s, %d of uint8 are needed" % (reset.numel(), reset.dtype, gr.N))
    _check(lib.rslx_gated_recurrence_step(gr.c, gr.view("x", x), gr.view("g", g), _ptr(reset), gr.state("s_in", s_in), gr.state("s_out", s_out),
                                          gr.view("h", h), _stream()), "rslx_gated_recurrence_step")


def rslx_rms_norm(x, residual, weight, eps, total, y, rstd):
    """x, y [rows, cols], residual and total (x + residual, written) likewise or None; weight [cols] and rstd [rows] float32 or None."""
    code, dtype, shape = _matrix("x", x)
    rows, cols = shape
    (px, ldx), (pr, ldr) = _rows("x", x, dtype, shape), _rows("residual", residual, dtype, shape)
    (pt, ldt), (py, ldy) = _rows("total", total, dtype, shape), _rows("y", y, dtype, shape)
    _check(lib.rslx_rms_norm(code, px, ldx, pr, ldr, rows, cols, _f32("weight", weight, cols), eps, pt, ldt, py, ldy, _f32("rstd", rstd, rows),
                             _stream()), "rslx_rms_norm")


def rslx_rms_norm_e4m3(x, residual, weight, eps, total, y, scales, rstd):
    """As rslx_rms_norm with y in float8_e4m3fn and a scale for each row, scales [rows] float32: the output is scales[:, None] * y."""
    code, dtype, shape = _matrix("x", x)
    rows, cols = shape
    (px, ldx), (pr, ldr) = _rows("x", x, dtype, shape), _rows("residual", residual, dtype, shape)
    (pt, ldt), (py, ldy) = _rows("total", total, dtype, shape), _rows("y", y, torch.float8_e4m3fn, shape)
    _check(lib.rslx_rms_norm_e4m3(code, px, ldx, pr, ldr, rows, cols, _f32("weight", weight, cols), eps, pt, ldt, py, ldy,
                                  _f32("scales", scales, rows), _f32("rstd", rstd, rows), _stream()), "rslx_rms_norm_e4m3")


def rslx_rms_norm_backward_workspace_bytes(rows, cols):
    n = lib.rslx_rms_norm_backward_workspace_bytes(rows, _int32("cols", cols))
    if n == 0:
        raise RslxError("rslx_rms_norm_backward_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_rms_norm_backward(dy, total, weight, rstd, dtotal, dx, dweight, ws):
    """dy, total, dx [rows, cols], dtotal (the gradient of total) likewise or None; rstd [rows] as rslx_rms_norm leaves it; dx, dweight or None."""
    code, dtype, shape = _matrix("total", total)
    rows, cols = shape
    (pt, ldt), (pd, lddy) = _rows("total", total, dtype, shape), _rows("dy", dy, dtype, shape)
    (ps, lddt), (pg, lddx) = _rows("dtotal", dtotal, dtype, shape), _rows("dx", dx, dtype, shape)
    _check(lib.rslx_rms_norm_backward(code, pd, lddy, pt, ldt, rows, cols, _f32("weight", weight, cols), _f32("rstd", rstd, rows), ps, lddt, pg, lddx,
                                      _f32("dweight", dweight, cols), _ptr(ws), ws.numel() if ws is not None else 0, _stream()),
           "rslx_rms_norm_backward")


class Muon:
    """Matrices of a Muon step (struct rslx_muon_matrix) and its constants (struct rslx_muon_cfg).  `matrices`: tuples (w_in, w_out, grad, m_in, m_out,
    scale) of contiguous float32 [rows, cols] (views into flat parameter buffers among them); w_in, m_in and m_out may be None."""

    def __init__(self, matrices, lr, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5):
        self.matrices = [tuple(m) for m in matrices]
        self.c = (_CMuonMatrix * max(len(self.matrices), 1))()
        for i, (w_in, w_out, grad, m_in, m_out, scale) in enumerate(self.matrices):
            if grad is None or grad.dim() != 2:
                raise RslxError("Muon: grad of matrix %d is not a matrix" % i)
            for name, t in (("w_in", w_in), ("w_out", w_out), ("grad", grad), ("m_in", m_in), ("m_out", m_out)):
                if t is not None and (t.dtype is not torch.float32 or t.shape != grad.shape):
                    raise RslxError("Muon: %s of matrix %d is %s %s, float32 %s is needed" % (name, i, t.dtype, tuple(t.shape), tuple(grad.shape)))
            rows, cols = (_int32("a side of matrix %d" % i, n) for n in grad.shape)
            self.c[i] = _CMuonMatrix(_ptr(w_in), _ptr(w_out), _ptr(grad), _ptr(m_in), _ptr(m_out), rows, cols, scale)
        self.cfg = _CMuonCfg(lr, momentum, weight_decay, int(bool(nesterov)), _int32("steps", steps))


def rslx_muon_step_workspace_bytes(muon):
    n = lib.rslx_muon_step_workspace_bytes(muon.c, len(muon.matrices), muon.cfg)
    if n == 0:
        raise RslxError("rslx_muon_step_workspace_bytes: %s" % lib.rslx_last_error().decode())
    return n


def rslx_muon_step(muon, ws):
    """One step of every matrix; lr may be changed between steps (muon.cfg.lr)."""
    _check(lib.rslx_muon_step(muon.c, len(muon.matrices), muon.cfg, _ptr(ws), ws.numel() if ws is not None else 0, _stream()), "rslx_muon_step")


def rslx_trace_begin(max_records):
    _check(lib.rslx_trace_begin(max_records), "rslx_trace_begin")


def rslx_trace_end():
    """Returns [(kernel, flops, bytes, ms)] in launch order."""
    n = C.c_int32(0)
    _check(lib.rslx_trace_end(None, 0, C.byref(n)), "rslx_trace_end")
    buf = (_CTraceRecord * max(n.value, 1))()
    _check(lib.rslx_trace_end(buf, n.value, C.byref(n)), "rslx_trace_end")
    return [(buf[i].kernel.decode(), buf[i].flops, buf[i].bytes, buf[i].ms) for i in range(n.value)]
