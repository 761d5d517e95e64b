"""ctypes binding of include/bsr.h.  Argument marshalling only: tensors are torch CUDA tensors used
as device memory, the stream is torch's current HIP stream.  Same names as the C entry points."""
from __future__ import annotations

import collections
import ctypes as C
import functools
import os

MAX_BLOCKS = 16
BSR_BF16, BSR_FP32 = 0, 1
BSR_SUMS_CUT = 256
BSR_LOSS_CE, BSR_LOSS_MEAN_SQ = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))

BLOCK_FIELDS = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_proj", "b_proj",
                "ln2_g", "ln2_b", "w_fc1", "b_fc1", "w_fc2", "b_fc2")
STEM_FIELDS = ("w_patch", "b_patch", "cls", "pos")
HEAD_FIELDS = ("lnf_g", "lnf_b", "w_head", "b_head")


class BsrError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"bsr error {code}: {text}")
        self.code = code


class bsr_config(C.Structure):
    _fields_ = [("image_size", C.c_int32), ("patch_size", C.c_int32), ("in_chans", C.c_int32),
                ("tokens_in", C.c_int32), ("dim", C.c_int32), ("heads", C.c_int32),
                ("mlp_hidden", C.c_int32), ("depth", C.c_int32), ("num_classes", C.c_int32),
                ("max_batch", C.c_int32), ("n_drop", C.c_int32),
                ("drop_blocks", C.c_int32 * MAX_BLOCKS), ("keep_k", C.c_int32 * MAX_BLOCKS),
                ("keep_ratio", C.c_float), ("first_trainable_block", C.c_int32),
                ("dtype", C.c_int32), ("loss", C.c_int32), ("ln_eps", C.c_float),
                ("n_experts", C.c_int32), ("moe_top_k", C.c_int32), ("n_moe", C.c_int32),
                ("moe_blocks", C.c_int32 * MAX_BLOCKS),
                ("n_trainable", C.c_int32), ("trainable_blocks", C.c_int32 * MAX_BLOCKS),
                ("fuse_dropped", C.c_int32), ("fold_frozen_layernorm", C.c_int32)]


class bsr_tile_choice(C.Structure):
    _fields_ = [("rows", C.c_int32), ("out", C.c_int32), ("in_", C.c_int32), ("tile", C.c_int32),
                ("microseconds", C.c_float)]


class bsr_block_params(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in BLOCK_FIELDS] + [("w_router", C.c_void_p)]


class bsr_params(C.Structure):
    _fields_ = ([(f, C.c_void_p) for f in STEM_FIELDS] + [("blocks", bsr_block_params * MAX_BLOCKS)]
                + [(f, C.c_void_p) for f in HEAD_FIELDS])


def lib_path() -> str:
    return os.path.join(_HERE, "libbsr_hip.so")


_lib = None


def load_library():
    """Load libbsr_hip.so.  Fails loudly when it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: run `python -m paper_2405_10951_amd.build` "
                                "(or __graft_entry__.build()) first")
    lib = C.CDLL(path)
    lib.bsr_last_error.restype = C.c_char_p
    lib.bsr_last_error.argtypes = [C.c_void_p]
    for name in ("bsr_token_schedule", "bsr_workspace_bytes", "bsr_init", "bsr_refresh_weights",
                 "bsr_forward_frozen", "bsr_select_tokens", "bsr_train_blocks_fwd_bwd",
                 "bsr_sgd_step", "bsr_destroy", "bsr_profile_begin", "bsr_profile_end", "bsr_moe_routing_io",
                 "bsr_adamw_step", "bsr_saved_activation_bytes", "bsr_autotune", "bsr_autotune_overlapped",
                 "bsr_pipeline_step"):
        getattr(lib, name).restype = C.c_int32
    lib.bsr_token_schedule.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
    lib.bsr_saved_activation_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
    lib.bsr_init.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_void_p)]
    lib.bsr_refresh_weights.argtypes = [C.c_void_p, C.c_void_p]
    lib.bsr_forward_frozen.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_select_tokens.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                      C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_train_blocks_fwd_bwd.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                             C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_void_p]
    lib.bsr_sgd_step.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_float, C.c_float, C.c_void_p]
    lib.bsr_destroy.argtypes = [C.c_void_p]
    lib.bsr_moe_routing_io.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_adamw_step.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_float, C.c_float,
                                   C.c_float, C.c_float, C.c_int32, C.c_void_p]
    lib.bsr_autotune.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_tile_choices.restype = C.c_int32
    lib.bsr_tile_choices.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32]
    lib.bsr_autotune_overlapped.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_pipeline_step.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_float, C.c_float, C.c_float, C.c_void_p, C.c_void_p]
    lib.bsr_linear_forward.restype = C.c_int32
    lib.bsr_linear_forward.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                       C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
    lib.bsr_gemm_tile_shapes.restype = C.c_int32
    lib.bsr_gemm_tile_shapes.argtypes = [C.c_void_p, C.c_int32]
    lib.bsr_ln_linear_fold.restype = C.c_int32
    lib.bsr_ln_linear_fold.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_ln_linear_forward.restype = C.c_int32
    lib.bsr_ln_linear_forward.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_float, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p]
    lib.bsr_linear_dgrad.restype = C.c_int32
    lib.bsr_linear_dgrad.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
    lib.bsr_linear_wgrad.restype = C.c_int32
    lib.bsr_linear_wgrad.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    lib.bsr_linear_backward.restype = C.c_int32
    lib.bsr_linear_backward.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p]
    lib.bsr_linear_wgrad_static.restype = C.c_int32
    lib.bsr_linear_wgrad_static.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_attention_forward.restype = C.c_int32
    lib.bsr_attention_forward.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                          C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.bsr_attention_backward.restype = C.c_int32
    lib.bsr_attention_backward.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                           C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    p, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    for name, args in {
            "bsr_layernorm_forward": (p, i32, i64, i32, i64, p, p, f32, p, i64, p, p, p, p, p),
            "bsr_layernorm_backward": (p, i64, p, i64, p, i64, i32, i64, i32, p, p, p, p, i64, p, p, p, C.c_size_t, p),
            "bsr_rmsnorm_forward": (p, i64, p, i64, i32, i64, i32, p, f32, p, i64, p, i64, p, p, p, p),
            "bsr_rmsnorm_backward": (p, i64, p, i64, p, i64, i32, i64, i32, p, p, p, i64, p, p, C.c_size_t, p),
            "bsr_linear_ce_forward": (p, i64, p, i64, i32, i64, i32, i32, p, p, p, p, p, C.c_size_t, p),
            "bsr_linear_ce_backward": (p, i64, p, i64, i32, i64, i32, i32, p, p, p, p, f32, p, i64, p, i64, i32, p, p, C.c_size_t, p),
            "bsr_linear_ce_forward_backward": (p, i64, p, i64, i32, i64, i32, i32, p, p, p, p, f32, p, i64, p, i64, i32, p, p, C.c_size_t, p),
            "bsr_linear_ce_tiles": (i32, i64, i32, i32, i32, i32, p, i32),
            "bsr_clip_grads": (p, p, p, i32, f32, p, p, p, C.c_size_t, p),
            "bsr_quantize8_rows": (p, i32, i64, i32, i64, p, p, p),
            "bsr_quantize8_weight": (p, i32, i32, i32, i64, p, p, p, p, p),
            "bsr_linear8_forward": (p, i32, i64, p, i32, i32, i32, p, p, p, i32, p, p, p, i32, p, C.c_size_t, p),
            "bsr_linear8_dgrad": (p, i32, i64, p, i32, i32, i32, p, p, p, p, i32, p, C.c_size_t, p),
            "bsr_distill_forward": (p, i32, i64, i32, i64, p, i64, p, i32, i64, i32, p, f32, f32, p, p, p, f32, p, i64, p, C.c_size_t, p),
            "bsr_distill_backward": (p, i32, i64, i32, i64, p, i64, p, i32, i64, i32, p, f32, f32, p, p, f32, p, i64, p)}.items():
        getattr(lib, name).restype, getattr(lib, name).argtypes = i32, args
    lib.bsr_block8_strides.restype, lib.bsr_block8_strides.argtypes = None, (i32, p, p)
    lib.bsr_layernorm_workspace_floats.restype, lib.bsr_layernorm_workspace_floats.argtypes = C.c_size_t, (i32,)
    lib.bsr_rmsnorm_workspace_floats.restype, lib.bsr_rmsnorm_workspace_floats.argtypes = C.c_size_t, (i32,)
    lib.bsr_linear_ce_workspace_bytes.restype, lib.bsr_linear_ce_workspace_bytes.argtypes = C.c_size_t, (i32, i64, i32, i32, i32)
    lib.bsr_clip_workspace_bytes.restype, lib.bsr_clip_workspace_bytes.argtypes = C.c_size_t, (i32,)
    lib.bsr_distill_workspace_floats.restype, lib.bsr_distill_workspace_floats.argtypes = C.c_size_t, (i32, i64, i32)
    lib.bsr_linear8_workspace_bytes.restype, lib.bsr_linear8_workspace_bytes.argtypes = C.c_size_t, (i32, i32)
    lib.bsr_profile_begin.argtypes = [C.c_void_p]
    lib.bsr_profile_end.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    _lib = lib
    return lib


def make_config(cfg: dict, max_batch: int, keep_k=None) -> bsr_config:
    """Fill a bsr_config from a plain dict (the keys of the C struct; `first_trainable` is accepted
    for first_trainable_block, dtype may be "bf16"/"fp32")."""
    c = bsr_config()
    for f in ("image_size", "patch_size", "in_chans", "tokens_in", "dim", "heads", "mlp_hidden",
              "depth", "num_classes", "loss"):
        setattr(c, f, int(cfg.get(f, 0)))
    c.max_batch = int(max_batch)
    c.first_trainable_block = int(cfg.get("first_trainable_block", cfg.get("first_trainable", 0)))
    dt = cfg.get("dtype", "bf16")
    c.dtype = {"bf16": BSR_BF16, "fp32": BSR_FP32}.get(dt, dt)
    c.keep_ratio = float(cfg.get("keep_ratio", 1.0))
    c.ln_eps = float(cfg.get("ln_eps", 1e-6))
    drops = list(cfg.get("drop_blocks", []))
    c.n_drop = len(drops)
    for i, b in enumerate(drops):
        c.drop_blocks[i] = int(b)
    if keep_k is None:
        keep_k = cfg.get("keep_k")
    if keep_k:
        for i, k in enumerate(keep_k):
            c.keep_k[i] = int(k)
    moe = list(cfg.get("moe_blocks", []))
    c.n_moe = len(moe)
    for i, b in enumerate(moe):
        c.moe_blocks[i] = int(b)
    c.n_experts = int(cfg.get("n_experts", 0))
    c.moe_top_k = int(cfg.get("moe_top_k", 0))
    c.fuse_dropped = int(bool(cfg.get("fuse_dropped", 0)))
    c.fold_frozen_layernorm = int(bool(cfg.get("fold_frozen_layernorm", 0)))
    tb = list(cfg.get("trainable_blocks") or [])
    c.n_trainable = len(tb)
    for i, b in enumerate(tb):
        c.trainable_blocks[i] = int(b)
    if tb:
        c.first_trainable_block = int(tb[0])
    return c


def _check(rc, ctx=None):
    if rc != 0:
        raise BsrError(rc, load_library().bsr_last_error(ctx).decode())


def bsr_token_schedule(cfg: bsr_config):
    """-> (keep_k per drop, tokens seen by MHSA per block, tokens seen by the FFN per block)."""
    lib = load_library()
    kk = (C.c_int32 * MAX_BLOCKS)()
    ta = (C.c_int32 * MAX_BLOCKS)()
    tm = (C.c_int32 * MAX_BLOCKS)()
    _check(lib.bsr_token_schedule(C.byref(cfg), kk, ta, tm))
    return list(kk[:cfg.n_drop]), list(ta[:cfg.depth]), list(tm[:cfg.depth])


def bsr_workspace_bytes(cfg: bsr_config) -> int:
    n = C.c_size_t(0)
    _check(load_library().bsr_workspace_bytes(C.byref(cfg), C.byref(n)))
    return int(n.value)


class bsr_saved_bytes(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("qkv", "softmax", "attn_out", "gelu_in", "linear_in", "residual",
                                          "stats", "moe", "total")]


def bsr_saved_activation_bytes(cfg: bsr_config, batch: int):
    """-> (list per block of dict kind -> bytes, dict of sums) for `batch` images."""
    per = (bsr_saved_bytes * MAX_BLOCKS)()
    tot = bsr_saved_bytes()
    _check(load_library().bsr_saved_activation_bytes(C.byref(cfg), C.c_int32(batch), per, C.byref(tot)))
    as_dict = lambda r: {n: int(getattr(r, n)) for n, _ in bsr_saved_bytes._fields_}
    return [as_dict(per[l]) for l in range(cfg.depth)], as_dict(tot)


def _gpu_index(device):
    """Index of a GPU as torch gives it (None: the current one).  Refuses, as torch's own look-up of a stream does, a device that has
    none: the pointers that go with it would be host memory."""
    if device.type != "cuda":
        raise ValueError(f"tensors on a GPU are needed, these are on {device}")
    return device.index


def _raw_stream(index) -> int:
    """torch's current stream of a GPU, without the object around it.  The library launches on the current GPU: tensors on another one are refused."""
    import torch
    here = torch._C._cuda_getDevice()
    if index is not None and index != here:
        raise ValueError(f"tensors on cuda:{index}, the current GPU is cuda:{here} (torch.cuda.device or set_device)")
    return torch._C._cuda_getCurrentRawStream(here)


def _cur_stream(t):
    return _raw_stream(_gpu_index(t.device))


def bsr_linear_forward(x, w_t, bias=None, act=0, u_out=None, res=None, y=None, tile=0):
    """x [M,in] bf16, w_t [out,in] bf16 -> (y [M,out] bf16, used_mfma).  tile: 0 or a block-tile shape id."""
    import torch
    M, kin = x.shape
    out = w_t.shape[0]
    if y is None:
        y = torch.empty((M, out), dtype=torch.bfloat16, device=x.device)
    used = C.c_int32(-1)
    _check(load_library().bsr_linear_forward(_dp(x), M, kin, out, _dp(w_t), _dp(bias), act, _dp(u_out),
                                             _dp(res), _dp(y), tile, C.byref(used), _cur_stream(x)))
    return y, used.value


def bsr_gemm_tile_shapes():
    """Ids of the block-tile shapes of the bf16 product kernel."""
    lib = load_library()
    n = lib.bsr_gemm_tile_shapes(None, 0)
    ids = (C.c_int32 * n)()
    lib.bsr_gemm_tile_shapes(ids, n)
    return list(ids)


def bsr_ln_linear_fold(w, bias, gamma, beta):
    """w [in,out], bias [out], gamma [in], beta [in] fp32 -> (w_folded [out,in] bf16, colsum [out], bias_folded [out])."""
    import torch
    kin, out = w.shape
    wf = torch.empty((out, kin), dtype=torch.bfloat16, device=w.device)
    cs = torch.empty(out, dtype=torch.float32, device=w.device)
    bf = torch.empty(out, dtype=torch.float32, device=w.device)
    _check(load_library().bsr_ln_linear_fold(_dp(w), _dp(bias), _dp(gamma), _dp(beta), kin, out, _dp(wf), _dp(cs),
                                             _dp(bf), _cur_stream(w)))
    return wf, cs, bf


def bsr_ln_linear_forward(x, w_folded, colsum, bias_folded, eps=1e-6, act=0, tile=0, y=None):
    """x [M,in] bf16 and the folded tensors -> y [M,out] bf16 = act(LN(x) W + b)."""
    import torch
    M, kin = x.shape
    out = w_folded.shape[0]
    if y is None:
        y = torch.empty((M, out), dtype=torch.bfloat16, device=x.device)
    _check(load_library().bsr_ln_linear_forward(_dp(x), M, kin, out, _dp(w_folded), _dp(colsum), _dp(bias_folded),
                                                C.c_float(eps), act, _dp(y), tile, _cur_stream(x)))
    return y


def bsr_linear_dgrad(dy, w_s, u=None, dx=None, tile=0):
    """dy [M,out] bf16, w_s [in,out] bf16 -> (dx [M,in] bf16, used_mfma).  tile: 0 or a block-tile shape id."""
    import torch
    M, out = dy.shape
    kin = w_s.shape[0]
    if dx is None:
        dx = torch.empty((M, kin), dtype=torch.bfloat16, device=dy.device)
    used = C.c_int32(-1)
    _check(load_library().bsr_linear_dgrad(_dp(dy), M, kin, out, _dp(w_s), _dp(u), _dp(dx), tile, C.byref(used),
                                           _cur_stream(dy)))
    return dx, used.value


def bsr_linear_wgrad(x, dy, dw=None, workspace=None, db=None):
    """x [M,in], dy [M,out] bf16 -> (dw [in,out] fp32, used_mfma).  workspace: fp32 tensor or None;
    db: fp32 [out] tensor that receives the bias gradient, or None."""
    import torch
    M, kin = x.shape
    out = dy.shape[1]
    if dw is None:
        dw = torch.empty((kin, out), dtype=torch.float32, device=x.device)
    used = C.c_int32(-1)
    _check(load_library().bsr_linear_wgrad(_dp(x), _dp(dy), M, kin, out, _dp(dw), _dp(db), _dp(workspace),
                                           C.c_size_t(0 if workspace is None else workspace.numel()),
                                           C.byref(used), _cur_stream(x)))
    return dw, used.value


def bsr_linear_backward(x, dy, w_s, u=None, workspace=None, tile=0):
    """x [M,in], dy [M,out], w_s [in,out] bf16 -> (dx [M,in] bf16, dw [in,out] fp32, db [out] fp32), issued as the step issues
    them.  u [M,in]: dx is multiplied by GELU'(u)."""
    import torch
    M, kin = x.shape
    out = dy.shape[1]
    dx = torch.empty((M, kin), dtype=torch.bfloat16, device=x.device)
    dw = torch.empty((kin, out), dtype=torch.float32, device=x.device)
    db = torch.empty(out, dtype=torch.float32, device=x.device)
    _check(load_library().bsr_linear_backward(_dp(x), _dp(dy), M, kin, out, _dp(w_s), _dp(u), _dp(dx), _dp(dw), _dp(db), _dp(workspace),
                                              C.c_size_t(0 if workspace is None else workspace.numel()), tile, _cur_stream(x)))
    return dx, dw, db


def bsr_linear_wgrad_static(x, dy, dw=None, db=None):
    """bsr_linear_wgrad with the split-K partial sums in the library's built-in scratch array: the call itself
    allocates nothing (dw and db, when not given, are allocated here, in the binding)."""
    import torch
    M, kin = x.shape
    out = dy.shape[1]
    if dw is None:
        dw = torch.empty((kin, out), dtype=torch.float32, device=x.device)
    used = C.c_int32(-1)
    _check(load_library().bsr_linear_wgrad_static(_dp(x), _dp(dy), M, kin, out, _dp(dw), _dp(db), C.byref(used),
                                                  _cur_stream(x)))
    return dw, used.value


def bsr_attention_forward(qkv, heads, want_lse=True, want_cls=True):
    """qkv [B,T,3D] bf16 -> (out [B,T,D] bf16, lse [B,H,T] | None, cls_prob [B,H,T] | None, used_mfma)."""
    import torch
    B, T, D3 = qkv.shape
    D = D3 // 3
    out = torch.empty((B, T, D), dtype=torch.bfloat16, device=qkv.device)
    lse = torch.empty((B, heads, T), dtype=torch.float32, device=qkv.device) if want_lse else None
    cls = torch.empty((B, heads, T), dtype=torch.float32, device=qkv.device) if want_cls else None
    used = C.c_int32(-1)
    _check(load_library().bsr_attention_forward(_dp(qkv), B, T, heads, D // heads, _dp(out), _dp(lse), _dp(cls),
                                                C.byref(used), _cur_stream(qkv)))
    return out, lse, cls, used.value


def bsr_attention_backward(qkv, out, dout, lse, heads):
    """-> (dqkv [B,T,3D] bf16, used_mfma)."""
    import torch
    B, T, D3 = qkv.shape
    D = D3 // 3
    dqkv = torch.empty_like(qkv)
    delta = torch.empty((B, heads, T), dtype=torch.float32, device=qkv.device)
    used = C.c_int32(-1)
    _check(load_library().bsr_attention_backward(_dp(qkv), _dp(out), _dp(dout), _dp(lse), B, T, heads, D // heads,
                                                 _dp(delta), _dp(dqkv), C.byref(used), _cur_stream(qkv)))
    return dqkv, used.value


class Rows8:
    """Rows in 8 bits: `values` uint8 [M, ldv] (e4m3), `scales` uint8 [M, lds], contiguous, `cols` columns (see bsr.h).  Looked at where they are used."""
    __slots__ = ("values", "scales", "cols")

    def __init__(self, values, scales, cols):
        self.values, self.scales, self.cols = values, scales, int(cols)


class Weight8:
    """A frozen linear layer in 8 bits, laid out once: `values` / `scales` for the forward product, `values_back` / `scales_back`
    (None without) for the input gradient; n_in, n_out (see bsr.h).  Looked at once, here: its parts stay what they are."""
    __slots__ = ("values", "scales", "values_back", "scales_back", "n_in", "n_out")

    def __init__(self, values, scales, values_back, scales_back, n_in, n_out):
        import torch
        n_in, n_out = int(n_in), int(n_out)
        if n_in < 1 or n_out < 1 or (values_back is None) != (scales_back is None):
            raise ValueError(f"a layer of {n_in} inputs and {n_out} outputs, with values_back and scales_back or without both")
        for v, s, rows, cols, what in ((values, scales, n_out, n_in, ""), (values_back, scales_back, n_in, n_out, "_back")):
            if v is not None:
                ldv, lds = _block8_strides(cols)
                _flat(v, "values" + what, (rows, ldv), torch.uint8)
                _flat(s, "scales" + what, (-(-rows // 128), lds), torch.uint8)
                if v.device != values.device or s.device != values.device:
                    raise ValueError(f"tensors on {values.device}, {v.device} and {s.device}")
        for name, part in zip(self.__slots__, (values, scales, values_back, scales_back, n_in, n_out)):
            object.__setattr__(self, name, part)

    def __setattr__(self, name, value):
        raise AttributeError("the parts of a frozen layer are set when it is made")

    def __reduce__(self):                  # copies and pickles are made, and looked at, like the first one
        return Weight8, tuple(getattr(self, name) for name in self.__slots__)


# The operators on a caller's own tensors.  As everywhere in this module the library computes and nothing is recorded for autograd: results carry no graph, whether or not an argument
# asks for a gradient; gradients are what the backward calls return.
# The wrappers are on the path of calls that take the GPU a few microseconds, so what they look at they look at once and cheaply.
_types: dict = {}                  # torch type -> type code


def _type_code(t, what):
    if not _types:
        import torch
        _types.update({torch.bfloat16: BSR_BF16, torch.float32: BSR_FP32})
    code = _types.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: bfloat16 or float32 is needed, got {t.dtype}")
    return code


_LONGEST = 0x7fffffff              # of the lengths that the library takes in 32 bits, which would wrap around


def _in_32_bits(n, what):
    if n > _LONGEST:
        raise ValueError(f"{what}: {n}, at most {_LONGEST}")
    return n


def _rows_of(t, what, shape=None, dtype=None):
    """A tensor of two dimensions whose rows are contiguous -> its row stride."""
    s = t.shape
    if len(s) != 2 or (shape is not None and s != shape):
        raise ValueError(f"{what}: shape {tuple(s)}, {'two dimensions' if shape is None else tuple(shape)} expected")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{what}: {dtype} is needed, got {t.dtype}")
    ld, step = t.stride()
    cols = s[1]
    if cols > _LONGEST:
        _in_32_bits(cols, what + ": columns")
    if step != 1 and cols > 1:
        raise ValueError(f"{what}: the elements of a row have to lie together, stride {step}")
    if ld < cols:
        if s[0] > 1:
            raise ValueError(f"{what}: rows overlap (stride {ld}, {cols} columns)")
        ld = cols
    return ld


def _flat(t, what, shape, dtype):
    """The address of a contiguous tensor of a known shape and type."""
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {dtype} {tuple(shape)} expected, got {t.dtype} {tuple(t.shape)}, strides {t.stride()}")
    return t.data_ptr()


def _together(first, *others):
    """The current stream of the GPU that all tensors are on."""
    gpu = first.get_device()
    if gpu < 0:
        raise ValueError(f"tensors on a GPU are needed, these are on {first.device}")
    for t in others:
        if t is not None and t.get_device() != gpu:
            raise ValueError(f"tensors on {first.device} and {t.device}")
    return _raw_stream(gpu)


@functools.lru_cache(maxsize=256)
def _scratch_size(which, *sizes):
    """A size that the library names (a call costs as much as a look-up of a few of them)."""
    return getattr(load_library(), which)(*sizes)


def _like(t):
    """A new contiguous tensor of the shape and type of one."""
    if t.is_contiguous():
        import torch
        return torch.empty_like(t)
    return t.new_empty(t.shape)


def _block8_strides(cols):
    """bsr_block8_strides: of a row's values, of its scales"""
    nk = -(-cols // 128)
    return nk * 128, (nk + 3) // 4 * 4


def _rows8_new(M, K, like):
    import torch
    ldv, lds = _block8_strides(K)
    return Rows8(like.new_empty((M, ldv), dtype=torch.uint8), like.new_empty((M, lds), dtype=torch.uint8), K)


def bsr_quantize8_rows(x) -> Rows8:
    """x [M,K] bf16 or fp32 (any row stride) -> 8-bit rows, a scale for each 128 columns."""
    ld, code, stream = _rows_of(x, "x"), _type_code(x, "x"), _together(x)
    M, K = x.shape
    r = _rows8_new(M, K, x)
    _check(load_library().bsr_quantize8_rows(x.data_ptr(), code, M, K, ld, r.values.data_ptr(), r.scales.data_ptr(), stream))
    return r


def bsr_quantize8_weight(w, backward=True) -> Weight8:
    """w [in,out] bf16 or fp32 (any row stride) -> a frozen 8-bit layer, a scale for each 128 x 128; backward: with the copy that the input
    gradient reads."""
    ld, code = _rows_of(w, "w"), _type_code(w, "w")
    n_in, n_out = w.shape
    _in_32_bits(n_in, "w: rows")
    stream = _together(w)

    def new(rows, cols):
        import torch
        ldv, lds = _block8_strides(cols)
        return w.new_empty((rows, ldv), dtype=torch.uint8), w.new_empty((-(-rows // 128), lds), dtype=torch.uint8)

    v, s = new(n_out, n_in)
    vb, sb = new(n_in, n_out) if backward else (None, None)
    _check(load_library().bsr_quantize8_weight(_dp(w), code, n_in, n_out, ld, _dp(v), _dp(s), _dp(vb), _dp(sb), stream))
    return Weight8(v, s, vb, sb, n_in, n_out)


def _linear8(x, cols, what, *others):
    """-> (the rows' tensor, M, (pointer, type, stride, scales' pointer), workspace, its bytes, stream)"""
    if type(x) is Rows8:
        if x.cols != cols:
            raise ValueError(f"{what}: {x.cols} columns, the layer has {cols}")
        import torch
        t, u8 = x.values, torch.uint8
        M = _in_32_bits(t.shape[0], what + ": rows") if t.dim() else 0
        ldv, lds = _block8_strides(cols)
        p, s = _flat(t, what + ".values", (M, ldv), u8), _flat(x.scales, what + ".scales", (M, lds), u8)
        return t, M, (p, BSR_BF16, 0, s), None, 0, _together(t, x.scales, *others)
    ld = _rows_of(x, what)
    M, k = x.shape
    if k != cols:
        raise ValueError(f"{what}: {k} columns, the layer has {cols}")
    if M > _LONGEST:
        _in_32_bits(M, what + ": rows")
    stream = _together(x, *others)
    size, ws = _scratch_size("bsr_linear8_workspace_bytes", M, cols), None
    if size:
        import torch
        ws = x.new_empty(size, dtype=torch.uint8)
    return x, M, (x.data_ptr(), _type_code(x, what), ld, None), ws, size, stream


def _linear8_out(x, t, y, what, shape, out_dtype):
    if y is None:
        if out_dtype is None:
            if type(x) is not Rows8:
                return t.new_empty(shape)
            import torch
            out_dtype = torch.bfloat16
        return t.new_empty(shape) if t.dtype is out_dtype else t.new_empty(shape, dtype=out_dtype)
    if out_dtype is not None and y.dtype is not out_dtype:
        raise TypeError(f"{what}: {y.dtype}, out_dtype {out_dtype}")
    return y


def _linear8_type(t, what, cut_sums):
    """The result's type code, with how its sums are held."""
    code = _type_code(t, what)
    if not cut_sums:
        return code
    if code != BSR_BF16:
        raise ValueError(f"cut_sums: {what} in bfloat16 is needed, got {t.dtype}")
    return code | BSR_SUMS_CUT


def bsr_linear8_forward(x, w: Weight8, bias=None, act=0, u_out=None, res=None, y=None, out_dtype=None, cut_sums=False):
    """x [M,in] (Rows8, or bf16 / fp32 with any row stride) -> y [M,out] = act(x W + bias) (+ res), of out_dtype (that of x, bf16 for Rows8).
    act 1: GELU, u_out [M,out] receives its input.  cut_sums: faster sums of fewer bits for a bf16 result (BSR_SUMS_CUT in bsr.h)."""
    t, M, rows, ws, size, stream = _linear8(x, w.n_in, "x", w.values, bias, u_out, res, y)
    shape = (M, w.n_out)
    y = _linear8_out(x, t, y, "y", shape, out_dtype)
    if bias is not None:
        import torch
        _flat(bias, "bias", shape[1:], torch.float32)
    pu = None if u_out is None else _flat(u_out, "u_out", shape, y.dtype)
    pr = None if res is None else _flat(res, "res", shape, y.dtype)
    _check(load_library().bsr_linear8_forward(*rows, M, w.n_in, w.n_out, w.values.data_ptr(), w.scales.data_ptr(), _dp(bias), act, pu, pr,
                                              _flat(y, "y", shape, y.dtype), _linear8_type(y, "y", cut_sums), _dp(ws), size, stream))
    return y


def bsr_linear8_dgrad(dy, w: Weight8, u=None, dx=None, out_dtype=None, cut_sums=False):
    """dy [M,out] (Rows8, or bf16 / fp32 with any row stride) -> dx [M,in] = dy W^T, times GELU'(u) where u [M,in] is given.  cut_sums: as in
    bsr_linear8_forward."""
    if w.values_back is None:
        raise ValueError("the layer was laid out without backward")
    t, M, rows, ws, size, stream = _linear8(dy, w.n_out, "dy", w.values_back, u, dx)
    shape = (M, w.n_in)
    dx = _linear8_out(dy, t, dx, "dx", shape, out_dtype)
    pu = None if u is None else _flat(u, "u", shape, dx.dtype)
    _check(load_library().bsr_linear8_dgrad(*rows, M, w.n_in, w.n_out, w.values_back.data_ptr(), w.scales_back.data_ptr(), pu,
                                            _flat(dx, "dx", shape, dx.dtype), _linear8_type(dx, "dx", cut_sums), _dp(ws), size, stream))
    return dx


def _layernorm_forward(x, gamma, beta, eps, y, r8):
    ld, code, stream = _rows_of(x, "x"), _type_code(x, "x"), _together(x, gamma, beta, y)
    M, D = x.shape
    import torch
    f32 = torch.float32
    pg, pb = _flat(gamma, "gamma", (D,), f32), _flat(beta, "beta", (D,), f32)
    ldy = 0 if y is None else _rows_of(y, "y", x.shape, x.dtype)
    mean, rstd = gamma.new_empty(M), gamma.new_empty(M)
    pq, ps = (None, None) if r8 is None else (r8.values.data_ptr(), r8.scales.data_ptr())
    _check(load_library().bsr_layernorm_forward(x.data_ptr(), code, M, D, ld, pg, pb, eps, _dp(y), ldy, pq, ps, mean.data_ptr(),
                                                rstd.data_ptr(), stream))
    return mean, rstd


def bsr_layernorm_forward(x, gamma, beta, eps=1e-6, y=None):
    """x [M,D] bf16 or fp32 (any row stride), gamma, beta [D] fp32 -> (y [M,D], mean [M], rstd [M])."""
    if y is None:
        y = _like(x)
    mean, rstd = _layernorm_forward(x, gamma, beta, eps, y, None)
    return y, mean, rstd


def bsr_layernorm_forward8(x, gamma, beta, eps=1e-6, y=None):
    """The same with the result in 8 bits -> (Rows8, mean, rstd); y given: rounded to the type of x as well."""
    _rows_of(x, "x")
    r8 = _rows8_new(*x.shape, x)
    mean, rstd = _layernorm_forward(x, gamma, beta, eps, y, r8)
    return r8, mean, rstd


def bsr_layernorm_backward(dy, x, mean, rstd, gamma, res=None, dx=None, need_dx=True, need_params=True):
    """dy, x [M,D], mean, rstd [M] of the forward, gamma [D] -> (dx [M,D] | None, dgamma [D] | None, dbeta [D] | None).  res [M,D]: added to dx."""
    lib = load_library()
    ldx, code, stream = _rows_of(x, "x"), _type_code(x, "x"), _together(x, dy, mean, rstd, gamma, res, dx)
    shape, dtype = x.shape, x.dtype
    M, D = shape
    import torch
    f32 = torch.float32
    lddy = _rows_of(dy, "dy", shape, dtype)
    ldr = 0 if res is None else _rows_of(res, "res", shape, dtype)
    pm, ps, pg = _flat(mean, "mean", (M,), f32), _flat(rstd, "rstd", (M,), f32), _flat(gamma, "gamma", (D,), f32)
    if dx is None:
        lddx = D
        if need_dx:
            dx = _like(x)
    else:
        lddx = _rows_of(dx, "dx", shape, dtype)
    dg = db = ws = None
    floats = 0
    if need_params:
        floats = _scratch_size("bsr_layernorm_workspace_floats", D)
        dg, db, ws = gamma.new_empty(D), gamma.new_empty(D), gamma.new_empty(floats)
    _check(lib.bsr_layernorm_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, _dp(res), ldr, code, M, D, pm, ps, pg, _dp(dx), lddx, _dp(dg), _dp(db),
                                      _dp(ws), floats, stream))
    return dx, dg, db


def _rmsnorm_forward(x, gamma, eps, res, y, sum_out, r8):
    ldx, code, stream = _rows_of(x, "x"), _type_code(x, "x"), _together(x, gamma, res, y, sum_out)
    shape, dtype = x.shape, x.dtype
    M, D = shape
    import torch
    pg = _flat(gamma, "gamma", (D,), torch.float32)
    ldy = 0 if y is None else _rows_of(y, "y", shape, dtype)
    ldr = lds = 0
    if res is not None:
        ldr = _rows_of(res, "res", shape, dtype)
        if sum_out is None:
            sum_out, lds = _like(x), D
        else:
            lds = _rows_of(sum_out, "sum_out", shape, dtype)
    elif sum_out is not None:
        raise ValueError("sum_out is the sum of x and res, there is no res")
    rstd = gamma.new_empty(M)
    pq, ps = (None, None) if r8 is None else (r8.values.data_ptr(), r8.scales.data_ptr())
    _check(load_library().bsr_rmsnorm_forward(x.data_ptr(), ldx, _dp(res), ldr, code, M, D, pg, eps, _dp(sum_out), lds, _dp(y), ldy, pq, ps, rstd.data_ptr(), stream))
    return rstd, x if res is None else sum_out


def bsr_rmsnorm_forward(x, gamma, eps=1e-6, res=None, y=None, sum_out=None):
    """x, res [M,D] bf16 or fp32 (any row stride; res None: none), gamma [D] fp32 -> (y [M,D], rstd [M], what the norm is of: x + res [M,D], rounded once, or x itself)."""
    if y is None:
        y = _like(x)
    rstd, total = _rmsnorm_forward(x, gamma, eps, res, y, sum_out, None)
    return y, rstd, total


def bsr_rmsnorm_forward8(x, gamma, eps=1e-6, res=None, y=None, sum_out=None):
    """The same with the result in 8 bits -> (Rows8, rstd, x + res or x); y given: rounded to the type of x as well."""
    _rows_of(x, "x")
    r8 = _rows8_new(*x.shape, x)
    rstd, total = _rmsnorm_forward(x, gamma, eps, res, y, sum_out, r8)
    return r8, rstd, total


def bsr_rmsnorm_backward(dy, x, rstd, gamma, res=None, dx=None, need_dx=True, need_params=True):
    """dy [M,D], x [M,D] (what the norm was of), rstd [M] of the forward, gamma [D] -> (dx [M,D] | None, dgamma [D] | None).  res [M,D]: added to dx."""
    lib = load_library()
    ldx, code, stream = _rows_of(x, "x"), _type_code(x, "x"), _together(x, dy, rstd, gamma, res, dx)
    shape, dtype = x.shape, x.dtype
    M, D = shape
    import torch
    f32 = torch.float32
    lddy = _rows_of(dy, "dy", shape, dtype)
    ldr = 0 if res is None else _rows_of(res, "res", shape, dtype)
    ps, pg = _flat(rstd, "rstd", (M,), f32), _flat(gamma, "gamma", (D,), f32)
    if dx is None:
        lddx = D
        if need_dx:
            dx = _like(x)
    else:
        lddx = _rows_of(dx, "dx", shape, dtype)
    dg = ws = None
    floats = 0
    if need_params:
        floats = _scratch_size("bsr_rmsnorm_workspace_floats", D)
        dg, ws = gamma.new_empty(D), gamma.new_empty(floats)
    _check(lib.bsr_rmsnorm_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, _dp(res), ldr, code, M, D, ps, pg, _dp(dx), lddx, _dp(dg), _dp(ws), floats, stream))
    return dx, dg


def _distill_args(z, index, logits, labels, temperature, hard_weight):
    import torch
    ldz, code = _rows_of(z, "z"), _type_code(z, "z")
    rows, classes = z.shape
    shape = (rows, index.shape[-1])
    ldi = _rows_of(index, "index", shape, torch.int32)
    ldt = _rows_of(logits, "logits", shape)
    pl = None if labels is None else _flat(labels, "labels", (rows,), torch.int32)
    return (z.data_ptr(), code, rows, classes, ldz, index.data_ptr(), ldi, logits.data_ptr(), _type_code(logits, "logits"), ldt, shape[1], pl,
            temperature, hard_weight)


def _distill_dz(z, row_grad, dz):
    """-> (row_grad's address, dz, its row stride)"""
    pg = None
    if row_grad is not None:
        import torch
        pg = _flat(row_grad, "row_grad", z.shape[:1], torch.float32)
    if dz is None:
        return pg, _like(z), z.shape[1]
    return pg, dz, _rows_of(dz, "dz", z.shape, z.dtype)


def _distill_workspace(z, code):
    """-> (scratch of the forward or None, its floats)"""
    rows, classes = z.shape
    floats = _scratch_size("bsr_distill_workspace_floats", code, rows, classes)
    if not floats:
        return None, 0
    import torch
    return z.new_empty(floats, dtype=torch.float32), floats


def bsr_distill_forward(z, index, logits, labels=None, temperature=1.0, hard_weight=0.0):
    """Student logits z [rows,classes] bf16 or fp32, the teacher's classes index [rows,top] int32 (-1: absent) and logits [rows,top], labels
    [rows] int32 (-1: none) -> (loss [rows], stats [rows,3] for bsr_distill_backward)."""
    import torch
    stream = _together(z, index, logits, labels)
    args = _distill_args(z, index, logits, labels, temperature, hard_weight)
    loss, stats = z.new_empty(z.shape[0], dtype=torch.float32), z.new_empty((z.shape[0], 3), dtype=torch.float32)
    ws, floats = _distill_workspace(z, args[1])
    _check(load_library().bsr_distill_forward(*args, loss.data_ptr(), stats.data_ptr(), None, 1.0, None, 0, _dp(ws), floats, stream))
    return loss, stats


def bsr_distill_forward_backward(z, index, logits, labels=None, temperature=1.0, hard_weight=0.0, row_grad=None, grad_scale=1.0, dz=None):
    """-> (loss [rows], dz [rows,classes] = grad_scale row_grad[row] dloss/dz) in one pass.  dz may be z."""
    import torch
    stream = _together(z, index, logits, labels, row_grad, dz)
    args = _distill_args(z, index, logits, labels, temperature, hard_weight)
    pg, dz, ldd = _distill_dz(z, row_grad, dz)
    loss = z.new_empty(z.shape[0], dtype=torch.float32)
    ws, floats = _distill_workspace(z, args[1])
    _check(load_library().bsr_distill_forward(*args, loss.data_ptr(), None, pg, grad_scale, dz.data_ptr(), ldd, _dp(ws), floats, stream))
    return loss, dz


def bsr_distill_backward(z, index, logits, stats, row_grad=None, labels=None, temperature=1.0, hard_weight=0.0, grad_scale=1.0, dz=None):
    """dz [rows,classes] = grad_scale row_grad[row] dloss/dz from the stats of bsr_distill_forward.  dz may be z."""
    import torch
    stream = _together(z, index, logits, labels, stats, row_grad, dz)
    args = _distill_args(z, index, logits, labels, temperature, hard_weight)
    ps = _flat(stats, "stats", (z.shape[0], 3), torch.float32)
    pg, dz, ldd = _distill_dz(z, row_grad, dz)
    _check(load_library().bsr_distill_backward(*args, ps, pg, grad_scale, dz.data_ptr(), ldd, stream))
    return dz


def _linear_ce_args(x, w, labels, bias):
    """-> the arguments that both calls begin with"""
    import torch
    ldx, code = _rows_of(x, "x"), _type_code(x, "x")
    ldw = _rows_of(w, "w", dtype=x.dtype)
    rows, width = x.shape
    classes = w.shape[0]
    if w.shape[1] != width:
        raise ValueError(f"w: {w.shape[1]} columns, x has {width}")
    _in_32_bits(classes, "w: rows")
    pb = None if bias is None else _flat(bias, "bias", (classes,), torch.float32)
    return x.data_ptr(), ldx, w.data_ptr(), ldw, code, rows, width, classes, pb, _flat(labels, "labels", (rows,), torch.int32)


def _linear_ce_workspace(x, args, what):
    """-> (scratch or None, its bytes); torch's allocations are aligned to 512 bytes"""
    size = _scratch_size("bsr_linear_ce_workspace_bytes", *args[4:8], what)
    if not size:
        return None, 0
    import torch
    return x.new_empty(size, dtype=torch.uint8), size


def bsr_linear_ce_forward(x, w, labels, bias=None):
    """Cross-entropy of the logits x w^T + bias, which nobody keeps: x [rows,width] bf16 or fp32, w [classes,width] of the same type (any row strides), labels [rows] int32 (-1: the row
    counts for nothing), bias [classes] fp32 -> (loss [rows], stats [rows,2] for bsr_linear_ce_backward)."""
    import torch
    stream = _together(x, w, labels, bias)
    args = _linear_ce_args(x, w, labels, bias)
    rows, f32 = x.shape[0], torch.float32
    loss, stats = x.new_empty(rows, dtype=f32), x.new_empty((rows, 2), dtype=f32)
    ws, size = _linear_ce_workspace(x, args, 0)
    _check(load_library().bsr_linear_ce_forward(*args, loss.data_ptr(), stats.data_ptr(), _dp(ws), size, stream))
    return loss, stats


def _linear_ce_grads(x, w, bias, row_grad, dx, dw, need_dx, need_dw, need_db):
    """-> (dx, dw, db, row_grad's address, dx's, dx's stride, dw's address, dw's stride, dw's type code, db's address)"""
    import torch
    shape = x.shape
    pg = None if row_grad is None else _flat(row_grad, "row_grad", shape[:1], torch.float32)
    lddx = lddw = shape[1]
    if dx is not None:
        lddx = _rows_of(dx, "dx", shape, x.dtype)
    elif need_dx:
        dx = _like(x)
    if dw is not None:
        lddw = _rows_of(dw, "dw", w.shape)
    elif need_dw:
        dw = _like(w)
    db = None if bias is None or not need_db else bias.new_empty(bias.shape)
    return dx, dw, db, pg, _dp(dx), lddx, _dp(dw), lddw, 0 if dw is None else _type_code(dw, "dw"), _dp(db)


def bsr_linear_ce_backward(x, w, labels, stats, bias=None, row_grad=None, grad_scale=1.0, dx=None, dw=None, need_dx=True, need_dw=True, need_db=True):
    """The gradients of grad_scale * sum(row_grad * loss) (row_grad [rows] fp32, None: 1 for each) from the stats of the forward -> (dx [rows,width] | None, dw [classes,width] | None,
    db [classes] | None).  dw is of the type of w, or fp32 where a tensor of that type is given; there is no db without a bias."""
    import torch
    stream = _together(x, w, labels, bias, stats, row_grad, dx, dw)
    args = _linear_ce_args(x, w, labels, bias)
    ps = _flat(stats, "stats", (x.shape[0], 2), torch.float32)
    dx, dw, db, pg, *out = _linear_ce_grads(x, w, bias, row_grad, dx, dw, need_dx, need_dw, need_db)
    ws, size = _linear_ce_workspace(x, args, 1)
    _check(load_library().bsr_linear_ce_backward(*args, ps, pg, grad_scale, *out, _dp(ws), size, stream))
    return dx, dw, db


def bsr_linear_ce_forward_backward(x, w, labels, bias=None, row_grad=None, grad_scale=1.0, dx=None, dw=None, need_dx=True, need_dw=True, need_db=True):
    """-> (loss [rows], dx, dw, db) in one call."""
    import torch
    stream = _together(x, w, labels, bias, row_grad, dx, dw)
    args = _linear_ce_args(x, w, labels, bias)
    loss = x.new_empty(x.shape[0], dtype=torch.float32)
    dx, dw, db, pg, *out = _linear_ce_grads(x, w, bias, row_grad, dx, dw, need_dx, need_dw, need_db)
    ws, size = _linear_ce_workspace(x, args, 2)
    _check(load_library().bsr_linear_ce_forward_backward(*args, loss.data_ptr(), pg, grad_scale, *out, _dp(ws), size, stream))
    return loss, dx, dw, db


LinearCeTiles = collections.namedtuple("LinearCeTiles", "forward forward_pieces forward_last gradient pieces gradient_last products splits_x splits_w")


def bsr_linear_ce_tiles(rows, width, classes, dtype, aligned=True, dw_dtype=None):
    """How bsr_linear_ce_forward and bsr_linear_ce_backward go about such sizes (see include/bsr.h); host only."""
    code = {"bf16": BSR_BF16, "fp32": BSR_FP32}
    out = (C.c_int32 * len(LinearCeTiles._fields))()
    n = load_library().bsr_linear_ce_tiles(code[dtype], rows, width, classes, aligned, code[dw_dtype or dtype], out, len(out))
    _check(min(n, 0))
    return LinearCeTiles(*out)


def _clip_tensors(tensors, what):
    """-> (addresses, numbers of values, types) of contiguous tensors on one GPU.  (Lists through map: a call walks hundreds of tensors, and the GPU is done with ViT-B's in 55 us.)"""
    import torch
    t = torch.Tensor
    gpu = set(map(t.get_device, tensors))
    if len(gpu) != 1 or min(gpu) < 0:
        raise ValueError(f"{what}: tensors on one GPU are needed, these are on {sorted({str(g.device) for g in tensors})}")
    if not all(map(t.is_contiguous, tensors)):
        raise ValueError(f"{what}: contiguous tensors are needed")
    kinds = [g.dtype for g in tensors]
    for g in tensors if not _types or not _types.keys() >= set(kinds) else ():
        _type_code(g, what)
    return list(map(t.data_ptr, tensors)), list(map(t.numel, tensors)), kinds


def _clip(grads, max_norm, out):
    n = len(grads)
    if n == 0:
        raise ValueError("no gradients")
    at, lengths, kinds = _clip_tensors(grads, "gradients")
    first, to = grads[0], None
    gpu = first.get_device()
    if out is grads:
        to = at
    elif out is not None:
        if len(out) != n:
            raise ValueError(f"{n} gradients, {len(out)} results")
        to, more, same = _clip_tensors(out, "out")
        if more != lengths or same != kinds:
            raise ValueError("out: tensors of the gradients' types and numbers of values are needed")
        if out[0].get_device() != gpu:
            raise ValueError(f"tensors on {first.device} and {out[0].device}")
    import torch
    size = _scratch_size("bsr_clip_workspace_bytes", n)
    norm, ws = first.new_empty((), dtype=torch.float32), first.new_empty(size, dtype=torch.uint8)
    addresses = C.c_void_p * n
    _check(load_library().bsr_clip_grads(addresses(*at), (C.c_int32 * n)(*[_types[k] for k in kinds]), (C.c_int64 * n)(*lengths), n, max_norm,
                                         None if to is None else addresses(*to), norm.data_ptr(), ws.data_ptr(), size, _raw_stream(gpu)))
    return norm


def bsr_grad_norm(grads):
    """The norm of all gradients (a list of contiguous bf16 or fp32 tensors) taken together -> fp32 scalar on their GPU."""
    return _clip(list(grads), 0.0, None)


def bsr_clip_grads(grads, max_norm, out=None):
    """grads (a list of contiguous bf16 or fp32 tensors) times min(1, max_norm / their norm taken together), in place or to `out` (a list of contiguous tensors of
    as many values and the same types)
    -> the norm before, fp32 scalar on their GPU."""
    grads = list(grads)
    return _clip(grads, max_norm, grads if out is None else list(out))


_PointerTable = C.c_uint64 * (C.sizeof(bsr_params) // 8)       # a bsr_params, which holds nothing but pointers, by position
_position: dict = {}                                            # name of one of its tensors -> the position there


def _find_position(name: str) -> int:
    """-1: no tensor of that name in a bsr_params"""
    field, at = bsr_params, 0
    if name.startswith("blocks."):
        _, i, name = name.split(".")
        if not 0 <= int(i) < MAX_BLOCKS:
            raise IndexError(f"block {i}: at most {MAX_BLOCKS}")
        field, at = bsr_block_params, bsr_params.blocks.offset + int(i) * C.sizeof(bsr_block_params)
    if field is bsr_params and name == "blocks":
        raise TypeError("blocks: one tensor does not stand for all blocks")
    return (at + getattr(field, name).offset) // 8 if name in [f[0] for f in field._fields_] else -1


def _params_struct(tensors: dict):
    """The pointers as the library takes them.  (Field by field through ctypes, a name split and two objects made for every tensor,
    a one-block step spent 25 us of host time here, a quarter of what it takes on the GPU.)"""
    p = _PointerTable()
    for name, t in tensors.items():
        if t is None:
            continue
        at = _position.get(name)
        if at is None:
            at = _find_position(name)
            if at < 0:
                continue
            _position[name] = at          # (only names of the library's own: a bounded table)
        p[at] = t.data_ptr()
    return p


def _dp(t):
    return None if t is None else t.data_ptr()


class Context:
    """Owns a bsr_ctx and the torch tensors (device memory) it points into.  Methods carry the
    names of the C entry points and forward to them one to one."""

    def __init__(self, cfg: dict, params: dict, max_batch: int, keep_k=None, device="cuda:0"):
        import torch
        self.torch = torch
        self.lib = load_library()
        self.device = torch.device(device)
        self._gpu = _gpu_index(self.device)
        self.c = make_config(cfg, max_batch, keep_k)
        self.act_dtype = torch.float32 if self.c.dtype == BSR_FP32 else torch.bfloat16
        self.keep_k, self.tokens_attn, self.tokens_mlp = bsr_token_schedule(self.c)
        # master weights: fp32 device tensors owned here, updated in place by bsr_sgd_step
        self.params = {k: torch.as_tensor(v, dtype=torch.float32).to(self.device).contiguous()
                       for k, v in params.items()}
        self._pstruct = _params_struct(self.params)
        nbytes = bsr_workspace_bytes(self.c)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) & ~255
        self.ctx = C.c_void_p()
        _check(self.lib.bsr_init(C.byref(self.c), C.byref(self._pstruct), C.c_void_p(base),
                                 C.c_size_t(nbytes), self._stream(), C.byref(self.ctx)))
        ft, L = self.c.first_trainable_block, self.c.depth
        self.T_f = self.tokens_attn[ft] if ft < L else self.tokens_mlp[L - 1]
        self.T_last = self.tokens_mlp[L - 1]
        self.frozen_drops = [i for i in range(self.c.n_drop) if self.c.drop_blocks[i] < ft]
        self.train_drops = [i for i in range(self.c.n_drop) if self.c.drop_blocks[i] >= ft]
        tb = [self.c.trainable_blocks[i] for i in range(self.c.n_trainable)]
        self.trainable_names = [n for n in self.params if n in HEAD_FIELDS or
                                (n.startswith("blocks.") and
                                 ((int(n.split(".")[1]) in tb) if tb else int(n.split(".")[1]) >= ft))]

    def _stream(self):
        return _raw_stream(self._gpu)

    def _chk(self, rc):
        if rc:
            _check(rc, self.ctx)

    def n_in(self, drop_i: int) -> int:
        """patch tokens entering drop location drop_i"""
        return self.tokens_attn[self.c.drop_blocks[drop_i]] - 1

    def new_grads(self) -> dict:
        return {n: self.torch.zeros_like(self.params[n]) for n in self.trainable_names}

    def moe_rows(self, B: int) -> dict:
        """block -> number of token rows (B * tokens of its FFN) for every mixture-of-experts block"""
        return {self.c.moe_blocks[i]: B * self.tokens_mlp[self.c.moe_blocks[i]] for i in range(self.c.n_moe)}

    # ---- entry points ---------------------------------------------------------------------
    def bsr_moe_routing_io(self, forced_experts=None, experts_out=None, router_logits_out=None):
        """Device tensors laid out block after block over the mixture-of-experts blocks (see bsr.h);
        the context only keeps the pointers, so the tensors are kept alive here."""
        self._moe_io = (forced_experts, experts_out, router_logits_out)
        self._chk(self.lib.bsr_moe_routing_io(self.ctx, _dp(forced_experts), _dp(experts_out),
                                              _dp(router_logits_out)))

    def bsr_refresh_weights(self):
        self._chk(self.lib.bsr_refresh_weights(self.ctx, self._stream()))

    def bsr_forward_frozen(self, inp, x_out=None, kept_idx_out=None, scores_out=None, forced_idx=None):
        t = self.torch
        B = inp.shape[0]
        if x_out is None:
            x_out = t.empty((B, self.T_f, self.c.dim), dtype=self.act_dtype, device=self.device)
        self._chk(self.lib.bsr_forward_frozen(self.ctx, _dp(inp), B, _dp(x_out), _dp(kept_idx_out),
                                              _dp(scores_out), _dp(forced_idx), self._stream()))
        return x_out

    def bsr_select_tokens(self, cls_attn, x_in, k, idx_out=None, x_out=None):
        t = self.torch
        B, n = cls_attn.shape
        if idx_out is None:
            idx_out = t.empty((B, max(k, 1)), dtype=t.int32, device=self.device)
        if x_in is not None and x_out is None:
            x_out = t.empty((B, k + 1, self.c.dim), dtype=self.act_dtype, device=self.device)
        self._chk(self.lib.bsr_select_tokens(self.ctx, _dp(cls_attn), _dp(x_in), B, n, k, _dp(idx_out),
                                             _dp(x_out), self._stream()))
        return idx_out[:, :k], x_out

    def bsr_train_blocks_fwd_bwd(self, x_in, labels, grads: dict, loss_out=None, logits_out=None,
                                 x_final_out=None, kept_idx_out=None, scores_out=None, forced_idx=None):
        t = self.torch
        B = x_in.shape[0]
        if loss_out is None:
            loss_out = t.zeros(4, dtype=t.float32, device=self.device)
        gs = _params_struct(grads)
        self._chk(self.lib.bsr_train_blocks_fwd_bwd(self.ctx, _dp(x_in), _dp(labels), B, _dp(loss_out),
                                                    _dp(logits_out), _dp(x_final_out), C.byref(gs),
                                                    _dp(kept_idx_out), _dp(scores_out), _dp(forced_idx),
                                                    self._stream()))
        return loss_out

    def bsr_sgd_step(self, grads: dict, momenta: dict | None, lr: float, momentum: float = 0.0,
                     weight_decay: float = 0.0):
        gs = _params_struct(grads)
        ms = _params_struct(momenta) if momenta is not None else None
        self._chk(self.lib.bsr_sgd_step(self.ctx, C.byref(gs), C.byref(ms) if ms is not None else None,
                                        C.c_float(lr), C.c_float(momentum), C.c_float(weight_decay),
                                        self._stream()))

    def bsr_autotune(self, inp, labels, x_frozen, loss_out, grads: dict):
        """-> (launches with a measured tile choice, how many differ from the cost model's)."""
        gs = _params_struct(grads)
        n, ch = C.c_int32(0), C.c_int32(0)
        self._chk(self.lib.bsr_autotune(self.ctx, _dp(inp), _dp(labels), C.c_int32(inp.shape[0]), _dp(x_frozen),
                                        _dp(loss_out), C.byref(gs), C.byref(n), C.byref(ch), self._stream()))
        return int(n.value), int(ch.value)

    def bsr_tile_choices(self, part: int):
        """[(rows, out, in, tile, microseconds)] of the launches of part 0 (frozen prefix) or 1 (trainable part)."""
        n = self.lib.bsr_tile_choices(self.ctx, part, None, 0)
        buf = (bsr_tile_choice * max(n, 1))()
        self.lib.bsr_tile_choices(self.ctx, part, buf, n)
        return [(b.rows, b.out, b.in_, b.tile, b.microseconds) for b in buf[:n]]

    def bsr_pipeline_step(self, inp_next, x_next, x_cur, labels_cur, loss_out, grads: dict, momenta: dict | None, lr: float,
                          momentum: float, weight_decay: float, stream_frozen, stream_train):
        """Frozen prefix of the next batch (inp_next -> x_next, both None on the last step) on stream_frozen beside
        the trainable part + SGD step of the current batch (x_cur, None on the first call) on stream_train
        (two torch streams)."""
        gs = _params_struct(grads)
        ms = _params_struct(momenta) if momenta is not None else None
        B = (inp_next if inp_next is not None else x_cur).shape[0]
        self._chk(self.lib.bsr_pipeline_step(self.ctx, _dp(inp_next), _dp(x_next), _dp(x_cur), _dp(labels_cur), C.c_int32(B),
                                             _dp(loss_out), C.byref(gs), C.byref(ms) if ms is not None else None,
                                             C.c_float(lr), C.c_float(momentum), C.c_float(weight_decay),
                                             C.c_void_p(stream_frozen.cuda_stream), C.c_void_p(stream_train.cuda_stream)))

    def bsr_autotune_overlapped(self, inp, labels, x_frozen, x_side, loss_out, grads: dict, side_stream):
        """Tile choice timed with the frozen prefix (current stream) beside the trainable part (side_stream, a
        torch stream); -> (launches with a measured tile choice, how many differ from the cost model's)."""
        gs = _params_struct(grads)
        n, ch = C.c_int32(0), C.c_int32(0)
        self._chk(self.lib.bsr_autotune_overlapped(self.ctx, _dp(inp), _dp(labels), C.c_int32(inp.shape[0]), _dp(x_frozen),
                                                   _dp(x_side), _dp(loss_out), C.byref(gs), C.byref(n), C.byref(ch),
                                                   self._stream(), C.c_void_p(side_stream.cuda_stream)))
        return int(n.value), int(ch.value)

    def bsr_adamw_step(self, grads: dict, exp_avg: dict, exp_avg_sq: dict, lr: float, beta1: float = 0.9,
                       beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01, step: int = 1):
        gs, ms, vs = _params_struct(grads), _params_struct(exp_avg), _params_struct(exp_avg_sq)
        self._chk(self.lib.bsr_adamw_step(self.ctx, C.byref(gs), C.byref(ms), C.byref(vs), C.c_float(lr),
                                          C.c_float(beta1), C.c_float(beta2), C.c_float(eps),
                                          C.c_float(weight_decay), C.c_int32(step), self._stream()))

    def bsr_clip_grads(self, grads: dict, max_norm: float):
        """The trainable tensors' gradients brought down to a largest norm, all of them taken together, in place, for bsr_sgd_step or bsr_adamw_step
        behind it; -> the norm before (a scalar on the GPU)."""
        return bsr_clip_grads(list(grads.values()), max_norm)

    def bsr_profile_begin(self):
        self._chk(self.lib.bsr_profile_begin(self.ctx))

    def bsr_profile_end(self) -> dict:
        """-> {class: (ms, flops, launches)} for gemm / attn_fwd / attn_bwd; waits for the stream."""
        ms = (C.c_double * 3)()
        fl = (C.c_double * 3)()
        n = (C.c_int32 * 3)()
        self._chk(self.lib.bsr_profile_end(self.ctx, ms, fl, n))
        return {name: (ms[i], fl[i], n[i]) for i, name in enumerate(("gemm", "attn_fwd", "attn_bwd"))}

    def bsr_destroy(self):
        if self.ctx:
            self.lib.bsr_destroy(self.ctx)
            self.ctx = C.c_void_p()

    def __del__(self):
        try:
            self.bsr_destroy()
        except Exception:
            pass
