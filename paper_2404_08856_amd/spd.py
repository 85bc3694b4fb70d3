"""ctypes binding of libspd (argument marshalling only; every step runs in the HIP kernels).

Function names and arguments mirror include/spd.h.  torch is used for device memory
and the current stream, nothing else.  There is no fallback: if the shared library
has not been built, importing this module raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspd.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_2404_08856_amd.build, "
                      "or __graft_entry__.build()); there is no CPU fallback")
_lib = ctypes.CDLL(LIB_PATH)

SPD_OK = 0
SPD_ERR_INVALID_ARG, SPD_ERR_SHAPE, SPD_ERR_CAPACITY, SPD_ERR_HIP = -1, -2, -3, -4
SPD_TARGET_IS_PROBS, SPD_DRAFT_IS_PROBS = 1, 2
SPD_ROWS_ARE_PROBS = SPD_W_IS_BF16 = SPD_X_IS_BF16 = 1
SPD_ROPE_INVERSE = 2
SPD_ROPE_NONE, SPD_ROPE_LINEAR, SPD_ROPE_RAMP, SPD_ROPE_LOG_RAMP = range(4)
SPD_MAX_ROWS, SPD_MAX_M, SPD_MAX_TOP = 64, 8, 32
SPD_MAX_HEAD_DIM, SPD_MAX_PAGED_SEQS, SPD_MAX_PAGED_ROWS, SPD_MAX_PAGED_HEADS, SPD_MAX_PAGED_POSITIONS, SPD_MAX_PAGED_ROW_HEADS = 256, 4096, 1 << 20, 1024, 1 << 30, 1 << 27

EXPORTS = ["spd_last_error", "spd_model_bytes", "spd_model_create", "spd_model_destroy", "spd_kv_set_len",
           "spd_kv_get_len", "spd_prefill", "spd_prefill_tokens", "spd_verify_forward", "spd_draft_step",
           "spd_accept_workspace_bytes", "spd_speculative_accept", "spd_trace_enable", "spd_trace_read",
           "spd_model_set_tuning", "spd_kv_lens_to_device", "spd_kv_lens_from_device", "spd_draft_step_strided",
           "spd_block_finish", "spd_device_status", "spd_speculative_accept_static", "spd_kv_export", "spd_probe_read_chain",
           "spd_model_bytes_q4", "spd_model_create_q4", "spd_q4_bytes", "spd_q4_quantize", "spd_q4_dequantize", "spd_q4_pack",
           "spd_q4_matmul_workspace_bytes", "spd_q4_matmul", "spd_logprobs_workspace_bytes", "spd_token_logprobs",
           "spd_rope_table_bytes", "spd_rope_table", "spd_rope_apply", "spd_paged_append", "spd_paged_attention_workspace_bytes", "spd_paged_attention",
           "spd_verify_paged_workspace_bytes", "spd_verify_forward_paged"]
TRACE_KINDS = ["qkv", "o", "gate_up", "down", "lm_head", "attention", "embed"]
PROJECTIONS = ["qkv", "o", "gate_up", "down", "lm_head"]


class SpdError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libspd error {code}: {msg}")
        self.code = code


class spd_model_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float),
                ("tied_embeddings", ctypes.c_int32), ("max_seqs", ctypes.c_int32),
                ("max_positions", ctypes.c_int32)]


class spd_tuning(ctypes.Structure):
    _fields_ = [("separate_qkv_attention", ctypes.c_int32), ("attention_slices", ctypes.c_int32),
                ("gemm_waves", ctypes.c_int32 * 5), ("gemm_grid_cap", ctypes.c_int32 * 5),
                ("gemm_general_kernel", ctypes.c_int32 * 5), ("gemm_ring", ctypes.c_int32 * 5), ("batch_kernel", ctypes.c_int32),
                ("wait_spin_limit", ctypes.c_uint32)]


_PP = ctypes.POINTER(ctypes.c_void_p)


class spd_weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("lm_head", ctypes.c_void_p), ("final_norm", ctypes.c_void_p),
                ("attn_norm", _PP), ("wq", _PP), ("wk", _PP), ("wv", _PP), ("wo", _PP),
                ("mlp_norm", _PP), ("w_gate", _PP), ("w_up", _PP), ("w_down", _PP)]


class spd_q4_matrix(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


_QP = ctypes.POINTER(spd_q4_matrix)


class spd_weights_q4(ctypes.Structure):
    _fields_ = [("group", ctypes.c_int32), ("embed", ctypes.c_void_p), ("lm_head", spd_q4_matrix), ("final_norm", ctypes.c_void_p),
                ("attn_norm", _PP), ("wq", _QP), ("wk", _QP), ("wv", _QP), ("wo", _QP),
                ("mlp_norm", _PP), ("w_gate", _QP), ("w_up", _QP), ("w_down", _QP)]


class spd_rope_config(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int32), ("theta", ctypes.c_float), ("factor", ctypes.c_float), ("low", ctypes.c_float),
                ("high", ctypes.c_float), ("original_positions", ctypes.c_float), ("magnitude", ctypes.c_float), ("h_factors", ctypes.POINTER(ctypes.c_float))]


class spd_rope(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class spd_heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_size_t), ("head_stride", ctypes.c_size_t)]


class spd_paged_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("e4m3", ctypes.c_int32)]


class spd_paged_batch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("table_stride", ctypes.c_size_t),
                ("page_table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("row_start", ctypes.c_void_p)]


_vp, _i32, _f32, _u32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_uint32, ctypes.c_size_t
_szp = ctypes.POINTER(ctypes.c_size_t)
_lib.spd_last_error.restype = ctypes.c_char_p
_lib.spd_last_error.argtypes = []
_lib.spd_model_bytes.argtypes = [ctypes.POINTER(spd_model_config), _szp, _szp, _szp]
_lib.spd_model_create.argtypes = [ctypes.POINTER(spd_model_config), ctypes.POINTER(spd_weights), _vp, _sz, _vp, _sz,
                                  _vp, _sz, _vp, ctypes.POINTER(_vp)]
_lib.spd_model_destroy.argtypes = [_vp]
_lib.spd_model_set_tuning.argtypes = [_vp, ctypes.POINTER(spd_tuning)]
_lib.spd_kv_set_len.argtypes = [_vp, ctypes.POINTER(_i32), _i32]
_lib.spd_kv_get_len.argtypes = [_vp, ctypes.POINTER(_i32), _i32]
_lib.spd_kv_export.argtypes = [_vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp]
_lib.spd_prefill.argtypes = [_vp, _i32, _vp, _i32, _vp, _vp]
_lib.spd_prefill_tokens.argtypes = [_vp, _i32, _vp, _i32, _vp, _vp]
_lib.spd_verify_forward.argtypes = [_vp, _vp, _i32, _i32, _vp, _vp]
_lib.spd_draft_step.argtypes = [_vp, _vp, _i32, _i32, _f32, _vp, _vp, _vp, _vp]
_lib.spd_accept_workspace_bytes.argtypes = [_i32, _i32, _i32, _szp]
_lib.spd_speculative_accept.argtypes = [_vp, _vp, _vp, _vp, _i32, _i32, _i32, _f32, _u32, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.spd_speculative_accept_static.argtypes = [_vp, _vp, _vp, _vp, _i32, _i32, _i32, _f32, _u32, _vp, _vp, _vp, _vp]
_lib.spd_probe_read_chain.argtypes = [_vp, _sz, _szp, _i32, _i32, _vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), _vp]
_lib.spd_trace_enable.argtypes = [_vp, _i32]
_lib.spd_trace_read.argtypes = [_vp, _i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_i32)]
_lib.spd_kv_lens_to_device.argtypes = [_vp, _vp]
_lib.spd_kv_lens_from_device.argtypes = [_vp, _vp]
_lib.spd_device_status.argtypes = [_vp, _vp]
_lib.spd_draft_step_strided.argtypes = [_vp, _vp, _i32, _i32, _i32, _f32, _vp, _i32, _vp, _sz, _vp, _i32, _vp]
_lib.spd_block_finish.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _f32, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _sz, _vp]
_lib.spd_model_bytes_q4.argtypes = [ctypes.POINTER(spd_model_config), _i32, _szp, _szp, _szp]
_lib.spd_model_create_q4.argtypes = [ctypes.POINTER(spd_model_config), ctypes.POINTER(spd_weights_q4), _vp, _sz, _vp, _sz,
                                     _vp, _sz, _vp, ctypes.POINTER(_vp)]
_lib.spd_q4_bytes.argtypes = [_i32, _i32, _i32, _szp]
_lib.spd_q4_quantize.argtypes = [_vp, _sz, _u32, _i32, _i32, _i32, _vp, _vp, _vp]
_lib.spd_q4_dequantize.argtypes = [_vp, _vp, _i32, _i32, _i32, _vp, _sz, _u32, _vp]
_lib.spd_q4_pack.argtypes = [_vp, _vp, _i32, _i32, _i32, _vp, _sz, _vp]
_lib.spd_q4_matmul_workspace_bytes.argtypes = [_i32, _i32, _i32, _szp]
_lib.spd_q4_matmul.argtypes = [_vp, _i32, _i32, _i32, _vp, _sz, _u32, _i32, _vp, _sz, _vp, _sz, _vp]
_lib.spd_logprobs_workspace_bytes.argtypes = [_i32, _i32, _i32, _szp]
_lib.spd_token_logprobs.argtypes = [_vp, _sz, _vp, _i32, _i32, _f32, _u32, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _sz, _vp]
_lib.spd_rope_table_bytes.argtypes = [_i32, _szp]
_lib.spd_rope_table.argtypes = [_vp, _vp, _sz, _vp]                    # (structures by address: byref objects as they are)
_lib.spd_rope_apply.argtypes = [_vp, _vp, _vp, _vp, _i32, _i32, _i32, _u32, _vp]
_lib.spd_paged_append.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _u32, _vp]
_lib.spd_paged_attention_workspace_bytes.argtypes = [_vp, _vp, _i32, _szp]
_lib.spd_paged_attention.argtypes = [_vp, _vp, _vp, _vp, _i32, _f32, _i32, _vp, _vp, _u32, _vp, _sz, _vp]
_lib.spd_verify_paged_workspace_bytes.argtypes = [_vp, _vp, _vp, _szp]
_lib.spd_verify_forward_paged.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
for _name in EXPORTS:
    if _name != "spd_last_error":
        getattr(_lib, _name).restype = _i32


def spd_last_error():
    return _lib.spd_last_error().decode()


def _check(rc):
    if rc != SPD_OK:
        raise SpdError(rc, spd_last_error())


# Pointers go to ctypes as plain integers, and the stream without a Python object around it: an accept call of one sequence was 12 us of this
# and one launch, more than its kernel takes.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device              # (no names that torch promises)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream():
    return _raw_stream(_current_device())


def _ptr(t, dtype=None):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device, contiguous tensors only"
    if dtype is not None:
        assert t.dtype == dtype, f"expected {dtype}, got {t.dtype}"
    return t.data_ptr()


def _raw(t, dtype):
    """Data pointer of a device tensor that may be a strided view into a larger buffer."""
    assert t.is_cuda and t.dtype == dtype
    return t.data_ptr()


# The smaller of the calls below take 3 to 8 us of device time: what is checked here is read from each tensor once.
_F32, _BF16, _I32, _U8 = torch.float32, torch.bfloat16, torch.int32, torch.uint8


def _matrix(t, device):
    """Data pointer, row stride and whether bfloat16, of a float32 or bfloat16 matrix on the current device with contiguous rows (a view into a wider buffer is fine)."""
    (n, k), (stride, step), dtype = t.shape, t.stride(), t.dtype
    assert t.get_device() == device and (dtype == _F32 or dtype == _BF16), f"expected float32 or bfloat16 on device {device}, got {dtype} on {t.device}"
    assert (step == 1 or k <= 1) and (stride >= k or n <= 1), f"contiguous rows that do not overlap only, got strides {t.stride()}"
    return t.data_ptr(), stride if n > 1 else k, 1 if dtype == _BF16 else 0


def _own(t, device, dtype, shape):
    """Data pointer of a contiguous tensor on the current device, of this type and shape (a tuple)."""
    if t is None:
        return None
    assert t.dtype == dtype and t.shape == shape and t.get_device() == device and t.is_contiguous(), \
        f"expected contiguous {dtype} {shape} on device {device}, got {t.dtype} {tuple(t.shape)} on {t.device}"
    return t.data_ptr()


def _scratch(workspace, device):
    """Data pointer and bytes of a workspace: contiguous uint8 on the current device."""
    assert workspace.dtype == _U8 and workspace.get_device() == device and workspace.is_contiguous(), "a workspace is uint8 on the current device"
    return workspace.data_ptr(), workspace.numel()


def make_config(shape, max_seqs, max_positions):
    """spd_model_config from a synth.ModelShape-like object."""
    return spd_model_config(shape.n_layers, shape.d_model, shape.n_heads, shape.head_dim, shape.d_ffn,
                            shape.vocab, shape.rms_eps, shape.rope_theta, int(shape.tied_embeddings),
                            max_seqs, max_positions)


def spd_model_bytes(cfg):
    p, k, w = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib.spd_model_bytes(ctypes.byref(cfg), ctypes.byref(p), ctypes.byref(k), ctypes.byref(w)))
    return p.value, k.value, w.value


def spd_model_bytes_q4(cfg, group):
    p, k, w = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib.spd_model_bytes_q4(ctypes.byref(cfg), group, ctypes.byref(p), ctypes.byref(k), ctypes.byref(w)))
    return p.value, k.value, w.value


def quantize_weights(weights, group=128):
    """Weights as produced by synth.make_weights with every matrix but the embedding table as a pair (q, scales) of
    spd_q4_quantize: what Model takes for a model in 4 bits.  With tied embeddings the LM head is the quantised table."""
    def q4(w):
        q = torch.empty((w.shape[0], (w.shape[1] + 1) // 2), dtype=torch.uint8, device=w.device)
        scales = torch.empty((w.shape[0], (w.shape[1] + group - 1) // group), dtype=torch.bfloat16, device=w.device)
        spd_q4_quantize(w, group, q, scales)
        return q, scales
    head = weights.get("lm_head")
    return {"group": group, "embed": weights["embed"], "lm_head": q4(weights["embed"] if head is None else head), "final_norm": weights["final_norm"],
            "layers": [{k: v if k.endswith("norm") else q4(v) for k, v in lw.items()} for lw in weights["layers"]]}


class Model:
    """Owns the three device buffers (torch allocations) and the spd_model handle."""

    def __init__(self, cfg, weights, device="cuda"):
        """weights: dict as produced by synth.make_weights, or by quantize_weights for a model in 4 bits, tensors on `device`."""
        self.cfg = cfg
        group = weights.get("group")
        pb, kb, wb = spd_model_bytes_q4(cfg, group) if group else spd_model_bytes(cfg)
        self.packed = torch.empty(pb, dtype=torch.uint8, device=device)
        self.kv = torch.zeros(kb, dtype=torch.uint8, device=device)
        self.workspace = torch.empty(wb, dtype=torch.uint8, device=device)
        L = cfg.n_layers
        assert len(weights["layers"]) == L

        def arr(key, dtype):
            a = (ctypes.c_void_p * L)()
            for l, lw in enumerate(weights["layers"]):
                a[l] = _ptr(lw[key], dtype)
            return a

        bf, f32 = torch.bfloat16, torch.float32
        handle = ctypes.c_void_p()
        if group:
            d, hd, F, V, here = cfg.d_model, cfg.n_heads * cfg.head_dim, cfg.d_ffn, cfg.vocab, _current_device()
            shapes = {"wq": (hd, d), "wk": (hd, d), "wv": (hd, d), "wo": (d, hd), "w_gate": (F, d), "w_up": (F, d), "w_down": (d, F)}

            def matrix(pair, n, k):
                return spd_q4_matrix(_own(pair[0], here, torch.uint8, (n, (k + 1) // 2)), _own(pair[1], here, bf, (n, (k + group - 1) // group)))
            mats = {key: (spd_q4_matrix * L)(*[matrix(lw[key], *shapes[key]) for lw in weights["layers"]]) for key in shapes}
            norms = [arr("attn_norm", f32), arr("mlp_norm", f32)]
            w = spd_weights_q4(group, _ptr(weights["embed"], bf), matrix(weights["lm_head"], V, d), _ptr(weights["final_norm"], f32),
                               ctypes.cast(norms[0], _PP), *[ctypes.cast(mats[k], _QP) for k in ("wq", "wk", "wv", "wo")],
                               ctypes.cast(norms[1], _PP), *[ctypes.cast(mats[k], _QP) for k in ("w_gate", "w_up", "w_down")])
            _check(_lib.spd_model_create_q4(ctypes.byref(cfg), ctypes.byref(w), _ptr(self.packed), pb, _ptr(self.kv), kb,
                                            _ptr(self.workspace), wb, _stream(), ctypes.byref(handle)))
            self.handle = handle
            torch.cuda.current_stream().synchronize()     # re-tiling done: the caller may drop `weights`
            return
        keep = [arr("attn_norm", f32), arr("wq", bf), arr("wk", bf), arr("wv", bf), arr("wo", bf),
                arr("mlp_norm", f32), arr("w_gate", bf), arr("w_up", bf), arr("w_down", bf)]
        w = spd_weights(_ptr(weights["embed"], bf), _ptr(weights.get("lm_head"), bf), _ptr(weights["final_norm"], f32),
                        *[ctypes.cast(a, _PP) for a in keep])
        _check(_lib.spd_model_create(ctypes.byref(cfg), ctypes.byref(w), _ptr(self.packed), pb, _ptr(self.kv), kb,
                                     _ptr(self.workspace), wb, _stream(), ctypes.byref(handle)))
        self.handle = handle
        torch.cuda.current_stream().synchronize()     # re-tiling done: the caller may drop `weights`

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:      # _lib is gone at interpreter shutdown
            _lib.spd_model_destroy(self.handle)
        self.handle = None

    def __del__(self):
        self.close()

    # --- thin wrappers, same names as the C entry points ---------------------------------
    def spd_model_set_tuning(self, separate_qkv_attention=0, attention_slices=0, gemm_waves=None, gemm_grid_cap=None,
                             gemm_general_kernel=None, gemm_ring=None, batch_kernel=0, wait_spin_limit=0):
        """Kernel-selection knobs for tests and sweeps; the per-projection dicts are keyed by PROJECTIONS."""
        t = spd_tuning()
        t.separate_qkv_attention, t.attention_slices, t.wait_spin_limit = int(separate_qkv_attention), int(attention_slices), int(wait_spin_limit)
        t.batch_kernel = int(batch_kernel)
        for field, given in (("gemm_waves", gemm_waves), ("gemm_grid_cap", gemm_grid_cap), ("gemm_general_kernel", gemm_general_kernel),
                             ("gemm_ring", gemm_ring)):
            for name, value in (given or {}).items():
                getattr(t, field)[PROJECTIONS.index(name)] = int(value)
        _check(_lib.spd_model_set_tuning(self.handle, ctypes.byref(t)))

    def spd_kv_set_len(self, lens):
        a = (ctypes.c_int32 * len(lens))(*[int(x) for x in lens])
        _check(_lib.spd_kv_set_len(self.handle, a, len(lens)))

    def spd_kv_get_len(self, n_seqs):
        a = (ctypes.c_int32 * n_seqs)()
        _check(_lib.spd_kv_get_len(self.handle, a, n_seqs))
        return list(a)

    def spd_kv_export(self, layer, seq, pos0, k_out, v_out):
        n = k_out.shape[0]
        assert k_out.shape == v_out.shape == (n, self.cfg.n_heads, self.cfg.head_dim)
        _check(_lib.spd_kv_export(self.handle, layer, seq, pos0, n, _ptr(k_out, torch.float32), _ptr(v_out, torch.float32), _stream()))

    def spd_prefill(self, seq, embeds, last_logits=None):
        _check(_lib.spd_prefill(self.handle, seq, _ptr(embeds, torch.float32), embeds.shape[0],
                                _ptr(last_logits, torch.float32), _stream()))

    def spd_prefill_tokens(self, seq, tokens, last_logits=None):
        _check(_lib.spd_prefill_tokens(self.handle, seq, _ptr(tokens, torch.int32), tokens.shape[0],
                                       _ptr(last_logits, torch.float32), _stream()))

    def spd_verify_forward(self, tokens, logits_out):
        n_seqs, M = tokens.shape
        assert logits_out.shape == (n_seqs, M, self.cfg.vocab)
        _check(_lib.spd_verify_forward(self.handle, _ptr(tokens, torch.int32), n_seqs, M,
                                       _ptr(logits_out, torch.float32), _stream()))

    def spd_verify_forward_paged(self, tokens, layers, batch, rope, logits_out, positions=None, seen=None, workspace=None):
        """tokens [batch.n_rows] through the model over pages: layers is a PagedCache per layer, logits_out [batch.n_rows, vocab]; seen (a tree) goes with positions."""
        here = _current_device()
        assert len(layers) == self.cfg.n_layers, f"expected {self.cfg.n_layers} layers, got {len(layers)}"
        assert all(c.device == here for c in layers) and batch.device == here and rope.device == here, f"pages, batch and table are on the current device {here}"
        pages, rows = (spd_paged_cache * len(layers))(*[c._struct for c in layers]), (batch.n_rows,)
        if workspace is None:
            b = ctypes.c_size_t()
            _check(_lib.spd_verify_paged_workspace_bytes(self.handle, pages, batch._at, ctypes.byref(b)))
            workspace = torch.empty(b.value, dtype=torch.uint8, device=tokens.device)
        _check(_lib.spd_verify_forward_paged(self.handle, _own(tokens, here, _I32, rows), pages, batch._at, rope._at, _own(positions, here, _I32, rows),
                                             _own(seen, here, _U64, rows), _own(logits_out, here, _F32, (batch.n_rows, self.cfg.vocab)), *_scratch(workspace, here), _raw_stream(here)))

    def spd_draft_step(self, tokens_in, temperature, u_draft, D_row_out, token_out):
        n_seqs, n_in = tokens_in.shape
        assert D_row_out.shape == (n_seqs, self.cfg.vocab) and token_out.shape == (n_seqs,) and u_draft.shape == (n_seqs,)
        _check(_lib.spd_draft_step(self.handle, _ptr(tokens_in, torch.int32), n_seqs, n_in, float(temperature),
                                   _ptr(u_draft, torch.float32), _ptr(D_row_out, torch.float32),
                                   _ptr(token_out, torch.int32), _stream()))


    def spd_draft_step_strided(self, tokens_in, in_stride, n_seqs, n_in, temperature, u_draft, u_stride,
                               D_row_out, D_stride, token_out, token_stride):
        """tokens_in, u_draft, D_row_out, token_out: device tensors (views into larger buffers are fine:
        only their data pointers are used; the strides are in elements between sequences)."""
        _check(_lib.spd_draft_step_strided(self.handle, _raw(tokens_in, torch.int32), in_stride, n_seqs, n_in,
                                           float(temperature), _raw(u_draft, torch.float32), u_stride,
                                           _raw(D_row_out, torch.float32), D_stride, _raw(token_out, torch.int32),
                                           token_stride, _stream()))

    def spd_device_status(self):
        _check(_lib.spd_device_status(self.handle, _stream()))

    def spd_kv_lens_to_device(self):
        _check(_lib.spd_kv_lens_to_device(self.handle, _stream()))

    def spd_kv_lens_from_device(self):
        _check(_lib.spd_kv_lens_from_device(self.handle, _stream()))

    def spd_trace_enable(self, enable):
        _check(_lib.spd_trace_enable(self.handle, int(bool(enable))))

    def spd_trace_read(self):
        """{kind: (milliseconds summed over launches, launches)} since the last read; waits for the events."""
        n = len(TRACE_KINDS)
        ms = (ctypes.c_double * n)()
        cnt = (ctypes.c_int32 * n)()
        _check(_lib.spd_trace_read(self.handle, n, ms, cnt))
        return {k: (ms[i], cnt[i]) for i, k in enumerate(TRACE_KINDS)}


def spd_block_finish(target, draft, target_logits, draft_probs, verify_tokens, u, temperature, n_accepted_out,
                     next_token_out, draft_in_out, out_tokens=None, n_out=None, workspace=None):
    n_seqs, g1, vocab = target_logits.shape
    gamma = g1 - 1
    assert draft_probs.shape == (n_seqs, gamma, vocab) and verify_tokens.shape == (n_seqs, g1) and u.shape == (n_seqs, g1)
    assert draft_in_out.shape == (n_seqs, 2)
    if workspace is None:
        workspace = torch.empty(spd_accept_workspace_bytes(n_seqs, gamma, vocab), dtype=torch.uint8, device=target_logits.device)
    cap = 0 if out_tokens is None else out_tokens.shape[1]
    _check(_lib.spd_block_finish(target.handle, draft.handle, _ptr(target_logits, torch.float32), _ptr(draft_probs, torch.float32),
                                 _ptr(verify_tokens, torch.int32), _ptr(u, torch.float32), n_seqs, gamma, float(temperature),
                                 _ptr(n_accepted_out, torch.int32), _ptr(next_token_out, torch.int32),
                                 _ptr(draft_in_out, torch.int32), _ptr(out_tokens, torch.int32), cap, _ptr(n_out, torch.int32),
                                 _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))
    return workspace


def spd_accept_workspace_bytes(n_seqs, gamma, vocab):
    b = ctypes.c_size_t()
    _check(_lib.spd_accept_workspace_bytes(n_seqs, gamma, vocab, ctypes.byref(b)))
    return b.value


def spd_speculative_accept(target, draft, draft_tokens, u, temperature, flags, n_accepted_out, next_token_out,
                           accept_prob_out=None, workspace=None):
    n_seqs, g1, vocab = target.shape
    gamma = g1 - 1
    assert draft.shape == (n_seqs, gamma, vocab) and draft_tokens.shape == (n_seqs, gamma) and u.shape == (n_seqs, g1)
    if workspace is None:
        workspace = torch.empty(spd_accept_workspace_bytes(n_seqs, gamma, vocab), dtype=torch.uint8, device=target.device)
    _check(_lib.spd_speculative_accept(_ptr(target, torch.float32), _ptr(draft, torch.float32),
                                       _ptr(draft_tokens, torch.int32), _ptr(u, torch.float32), n_seqs, gamma, vocab,
                                       float(temperature), int(flags), _ptr(n_accepted_out, torch.int32),
                                       _ptr(next_token_out, torch.int32), _ptr(accept_prob_out, torch.float32),
                                       _ptr(workspace), workspace.numel(), _stream()))


def spd_speculative_accept_static(target, draft, draft_tokens, u, temperature, flags, n_accepted_out, next_token_out,
                                  accept_prob_out=None):
    """spd_speculative_accept without a workspace argument (scratch memory inside the library); allocates nothing."""
    n_seqs, g1, vocab = target.shape
    gamma = g1 - 1
    assert draft.shape == (n_seqs, gamma, vocab) and draft_tokens.shape == (n_seqs, gamma) and u.shape == (n_seqs, g1)
    _check(_lib.spd_speculative_accept_static(_ptr(target, torch.float32), _ptr(draft, torch.float32),
                                              _ptr(draft_tokens, torch.int32), _ptr(u, torch.float32), n_seqs, gamma, vocab,
                                              float(temperature), int(flags), _ptr(n_accepted_out, torch.int32),
                                              _ptr(next_token_out, torch.int32), _ptr(accept_prob_out, torch.float32), _stream()))


def spd_logprobs_workspace_bytes(n_rows, vocab, n_top):
    b = ctypes.c_size_t()
    _check(_lib.spd_logprobs_workspace_bytes(n_rows, vocab, n_top, ctypes.byref(b)))
    return b.value


def spd_token_logprobs(rows, tokens, temperature, flags, logprob_out=None, entropy_out=None, rank_out=None, top_tokens_out=None,
                       top_logprobs_out=None, workspace=None):
    """rows [n, vocab] (a view into a wider buffer is fine); the number of alternatives is that of top_tokens_out's columns."""
    n, vocab = rows.shape
    here = _current_device()
    ptr, stride, bf16 = _matrix(rows, here)
    assert not bf16, "rows are float32"
    n_top = 0 if top_tokens_out is None else top_tokens_out.shape[1]
    if workspace is None:
        workspace = torch.empty(spd_logprobs_workspace_bytes(n, vocab, n_top), dtype=torch.uint8, device=rows.device)
    one, top = (n,), (n, n_top)
    _check(_lib.spd_token_logprobs(ptr, stride, _own(tokens, here, _I32, one), n, vocab, temperature, flags, _own(logprob_out, here, _F32, one),
                                   _own(entropy_out, here, _F32, one), _own(rank_out, here, _I32, one), n_top, _own(top_tokens_out, here, _I32, top),
                                   _own(top_logprobs_out, here, _F32, top), *_scratch(workspace, here), _raw_stream(here)))


def spd_q4_bytes(n, k, group):
    b = ctypes.c_size_t()
    _check(_lib.spd_q4_bytes(n, k, group, ctypes.byref(b)))
    return b.value


def spd_q4_quantize(w, group, q_out, scales_out):
    n, k = w.shape
    here = _current_device()
    ptr, stride, bf16 = _matrix(w, here)
    _check(_lib.spd_q4_quantize(ptr, stride, SPD_W_IS_BF16 * bf16, n, k, group, _own(q_out, here, torch.uint8, (n, (k + 1) // 2)),
                                _own(scales_out, here, torch.bfloat16, (n, (k + group - 1) // group)), _raw_stream(here)))


def spd_q4_dequantize(q, scales, group, w_out):
    n, k = w_out.shape
    here = _current_device()
    ptr, stride, bf16 = _matrix(w_out, here)
    _check(_lib.spd_q4_dequantize(_own(q, here, torch.uint8, (n, (k + 1) // 2)), _own(scales, here, torch.bfloat16, (n, (k + group - 1) // group)), n, k, group,
                                  ptr, stride, SPD_W_IS_BF16 * bf16, _raw_stream(here)))


class Q4Matrix:
    """A matrix [n, k] in 4 bits, laid out for spd_q4_matmul (owns the packed buffer; q and scales may be dropped)."""

    def __init__(self, q, scales, k, group):
        self.n, self.k, self.group = q.shape[0], int(k), int(group)
        self.packed = torch.empty(spd_q4_bytes(self.n, self.k, self.group), dtype=torch.uint8, device=q.device)
        here = _current_device()
        _check(_lib.spd_q4_pack(_own(q, here, torch.uint8, (self.n, (self.k + 1) // 2)), _own(scales, here, torch.bfloat16, (self.n, (self.k + self.group - 1) // self.group)),
                                self.n, self.k, self.group, *_scratch(self.packed, here), _raw_stream(here)))


def spd_q4_matmul_workspace_bytes(rows, n, k):
    b = ctypes.c_size_t()
    _check(_lib.spd_q4_matmul_workspace_bytes(rows, n, k, ctypes.byref(b)))
    return b.value


def spd_q4_matmul(matrix, x, y, workspace=None):
    """y [rows, matrix.n] float32 = x [rows, matrix.k] (float32 or bfloat16) times the matrix; both may be views into wider buffers."""
    rows, k = x.shape
    assert k == matrix.k and y.shape == (rows, matrix.n), f"expected [rows, {matrix.k}] and [rows, {matrix.n}], got {tuple(x.shape)} and {tuple(y.shape)}"
    here = _current_device()
    if workspace is None:
        workspace = torch.empty(spd_q4_matmul_workspace_bytes(rows, matrix.n, k), dtype=torch.uint8, device=x.device)
    packed = matrix.packed
    xp, xs, bf16 = _matrix(x, here)
    yp, ys, y_bf16 = _matrix(y, here)
    wp, wn = _scratch(workspace, here)
    assert packed.get_device() == here and not y_bf16, "the matrix is on the current device and y is float32"
    _check(_lib.spd_q4_matmul(packed.data_ptr(), matrix.n, k, matrix.group, xp, xs, SPD_X_IS_BF16 * bf16, rows, yp, ys, wp, wn, _raw_stream(here)))


# The handles below keep one ctypes structure each and its address as an integer: a paged call marshals plain numbers.
_U64 = torch.int64


def _heads(t, device, dtype):
    """Address of an spd_heads of a [rows, heads, dim] tensor on the current device whose heads' elements are neighbours (any strides between rows and heads)."""
    row, head, step = t.stride()
    assert t.dtype == dtype and t.get_device() == device and (step == 1 or t.shape[2] == 1), \
        f"expected {dtype} [rows, heads, dim] on device {device} with contiguous heads, got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}"
    return _byref(spd_heads(t.data_ptr(), row, head))


_byref = ctypes.byref


def _row_type(t):
    dtype = t.dtype
    assert dtype == _F32 or dtype == _BF16, f"expected float32 or bfloat16, got {dtype}"
    return dtype, SPD_X_IS_BF16 if dtype == _BF16 else 0


class Rope:
    """Rotary positions: the frequencies' table of spd_rope_table (owned) and how pairs lie in a head.  factors: one divisor per pair, or None."""

    def __init__(self, rotary_dim, theta=10000.0, interleaved=False, scaling=SPD_ROPE_NONE, factor=1.0, low=1.0, high=2.0, original_positions=1.0,
                 magnitude=1.0, factors=None, device="cuda"):
        b = ctypes.c_size_t()
        _check(_lib.spd_rope_table_bytes(rotary_dim, ctypes.byref(b)))
        assert factors is None or len(factors) == rotary_dim // 2, f"expected {rotary_dim // 2} factors"
        own = None if factors is None else (ctypes.c_float * len(factors))(*[float(f) for f in factors])
        cfg = spd_rope_config(rotary_dim, scaling, theta, factor, low, high, original_positions, magnitude, own)
        self.table = torch.empty(b.value, dtype=torch.uint8, device=device)
        here = _current_device()
        _check(_lib.spd_rope_table(ctypes.byref(cfg), *_scratch(self.table, here), _raw_stream(here)))
        self.rotary_dim, self.interleaved, self.device = int(rotary_dim), bool(interleaved), here
        self._struct = spd_rope(self.table.data_ptr(), self.rotary_dim, int(self.interleaved))
        self._at = ctypes.addressof(self._struct)


def spd_rope_apply(rope, x, positions, out, inverse=False):
    """out [rows, heads, dim] (x itself will do) = x turned by positions [rows] int32."""
    shape = x.shape
    rows, heads, dim = shape
    here = _current_device()
    dtype, flags = _row_type(x)
    assert out.shape == shape and rope.device == here, f"expected an output of {tuple(shape)}, and the table on device {here}"
    _check(_lib.spd_rope_apply(rope._at, _heads(x, here, dtype), _heads(out, here, dtype), _own(positions, here, _I32, (rows,)), rows, heads, dim,
                               flags | SPD_ROPE_INVERSE if inverse else flags, _raw_stream(here)))


def paged_cache_shapes(n_pages, page_size, n_kv_heads, head_dim, e4m3=False):
    """Shapes of the key and value tensors of a paged cache (bfloat16, or float8_e4m3fn)."""
    G = 16 if e4m3 else 8
    return (n_pages, n_kv_heads, head_dim // G, page_size, G), (n_pages, n_kv_heads, page_size // G, head_dim, G)


class PagedCache:
    """One layer's pages: k and v as paged_cache_shapes says, bfloat16, or float8_e4m3fn with a scale per head (kept, not copied)."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        e4m3 = k.dtype == torch.float8_e4m3fn
        here = k.get_device()
        n_pages, heads, granules, page_size, G = k.shape
        dim = granules * G
        assert k.dtype == (torch.float8_e4m3fn if e4m3 else _BF16), f"expected bfloat16 or float8_e4m3fn pages, got {k.dtype}"
        shapes = paged_cache_shapes(n_pages, page_size, heads, dim, e4m3)
        assert (k_scale is not None and v_scale is not None) == e4m3, "pages in e4m3 have scales, others none"
        self.k, self.v, self.k_scale, self.v_scale, self.device = k, v, k_scale, v_scale, here
        self.n_pages, self.page_size, self.n_kv_heads, self.head_dim, self.e4m3 = n_pages, page_size, heads, dim, e4m3
        self._struct = spd_paged_cache(_own(k, here, k.dtype, shapes[0]), _own(v, here, k.dtype, shapes[1]), _own(k_scale, here, _F32, (heads,)),
                                       _own(v_scale, here, _F32, (heads,)), n_pages, page_size, heads, dim, int(e4m3))
        self._at = ctypes.addressof(self._struct)


class PagedBatch:
    """The new rows of a paged call: page_table [n_seqs, max_pages] and lens [n_seqs] int32, row_start [n_seqs + 1] int32 or None (n_rows / n_seqs rows each).
    The tensors are kept, not copied: what they hold when a call runs counts."""

    def __init__(self, page_table, lens, n_rows, row_start=None):
        here = page_table.get_device()
        n_seqs, max_pages = page_table.shape
        stride, step = page_table.stride()
        assert page_table.dtype == _I32 and (step == 1 or max_pages <= 1) and (stride >= max_pages or n_seqs <= 1), "a page table is int32 with contiguous rows"
        self.page_table, self.lens, self.row_start, self.device = page_table, lens, row_start, here
        self.n_seqs, self.n_rows, self.max_pages = n_seqs, int(n_rows), max_pages
        self._struct = spd_paged_batch(n_seqs, self.n_rows, max_pages, stride if n_seqs > 1 else max_pages, page_table.data_ptr(),
                                       _own(lens, here, _I32, (n_seqs,)), _own(row_start, here, _I32, (n_seqs + 1,)))
        self._at = ctypes.addressof(self._struct)


def _paged_here(cache, batch):
    here = _current_device()
    assert cache.device == here and batch.device == here, f"the cache (device {cache.device}) and the batch ({batch.device}) are on the current device {here}"
    return here


def spd_paged_append(cache, batch, k, v, rope=None, positions=None, q=None, q_out=None):
    """k, v [n_rows, n_kv_heads, dim] into their places; with rope, k (and q [n_rows, heads, dim] into q_out) turned by positions, or by the rows' own."""
    here = _paged_here(cache, batch)
    rows, dim = batch.n_rows, cache.head_dim
    dtype, flags = _row_type(k)
    shape = (rows, cache.n_kv_heads, dim)
    assert k.shape == shape and v.shape == shape, f"expected keys and values {shape}, got {tuple(k.shape)} and {tuple(v.shape)}"
    qh = oh = None
    heads = 0
    if q is not None or q_out is not None:
        assert q is not None and q_out is not None, "q and q_out go together"
        heads = q.shape[1]
        assert q.shape == (rows, heads, dim) and q_out.shape == q.shape, f"expected queries [{rows}, heads, {dim}] and an output like them, got {tuple(q.shape)} and {tuple(q_out.shape)}"
        qh, oh = _heads(q, here, dtype), _heads(q_out, here, dtype)
    assert rope is None or rope.device == here, "the table is on the current device"
    _check(_lib.spd_paged_append(cache._at, batch._at, _heads(k, here, dtype), _heads(v, here, dtype), qh, oh, heads, None if rope is None else rope._at,
                                 None if positions is None else _own(positions, here, _I32, (rows,)), flags, _raw_stream(here)))


def spd_paged_attention_workspace_bytes(cache, batch, n_heads):
    b = ctypes.c_size_t()
    _check(_lib.spd_paged_attention_workspace_bytes(cache._at, batch._at, n_heads, ctypes.byref(b)))
    return b.value


def spd_paged_attention(cache, batch, q, out, scale=None, window=0, seen=None, lse_out=None, workspace=None):
    """out [n_rows, heads, dim] = attention of q over the rows' sequences; scale None: 1 / sqrt(dim); seen int64 [n_rows], the bits of new rows that a row sees."""
    here = _paged_here(cache, batch)
    rows, heads, dim = q.shape
    dtype, flags = _row_type(q)
    assert rows == batch.n_rows and dim == cache.head_dim and out.shape == q.shape, \
        f"expected queries [{batch.n_rows}, heads, {cache.head_dim}] and an output like them, got {tuple(q.shape)} and {tuple(out.shape)}"
    if workspace is None:
        workspace = torch.empty(spd_paged_attention_workspace_bytes(cache, batch, heads), dtype=torch.uint8, device=q.device)
    _check(_lib.spd_paged_attention(cache._at, batch._at, _heads(q, here, dtype), _heads(out, here, dtype), heads, dim ** -0.5 if scale is None else scale, window,
                                    _own(seen, here, _U64, (rows,)), _own(lse_out, here, _F32, (rows, heads)), flags, *_scratch(workspace, here), _raw_stream(here)))


def spd_probe_read_chain(buffer, stage_bytes, reps=20):
    """(per-kernel microseconds, microseconds per chain) of plain read kernels of the given sizes over `buffer` (a uint8 device tensor)."""
    n = len(stage_bytes)
    sizes = (ctypes.c_size_t * n)(*[int(b) for b in stage_bytes])
    sink = torch.zeros(1024, dtype=torch.int32, device=buffer.device)
    us = (ctypes.c_double * n)()
    chain = ctypes.c_double()
    _check(_lib.spd_probe_read_chain(_ptr(buffer, torch.uint8), buffer.numel(), sizes, n, int(reps), _ptr(sink), us, ctypes.byref(chain), _stream()))
    return list(us), chain.value
