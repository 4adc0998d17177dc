"""ctypes binding of libbf.so: argument marshalling only.  Every step of the path runs in
the library's HIP kernels; torch is used for device memory and streams.  There is no CPU
fallback: a missing library is an ImportError at load()."""
import ctypes as C
import os
from array import array as _array

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbf.so")

BF_OK, BF_EINVAL, BF_ENOMEM, BF_ESTATE, BF_EDEVICE = 0, -1, -2, -3, -4
BF_SCHED_BF, BF_SCHED_DF = 0, 1
BF_FP32, BF_BF16 = 0, 1
BF_CKPT_NONE, BF_CKPT_LAYER = 0, 1
BF_KERNELS_AUTO, BF_KERNELS_PLAIN = 0, 1
BF_NN, BF_NT, BF_TN = 0, 1, 2
BF_EPI_NONE, BF_EPI_BIAS, BF_EPI_BIAS_RES, BF_EPI_BIAS_GELU, BF_EPI_GELU_BWD, BF_EPI_ACCUM = range(6)
VOCAB_TENSOR_IDS = {"e_tok": 12, "e_pos": 13, "lnf_g": 14, "lnf_b": 15, "w_out": 16}
TENSOR_IDS = {"ln1_g": 0, "ln1_b": 1, "w_qkv": 2, "b_qkv": 3, "w_o": 4, "b_o": 5,
              "ln2_g": 6, "ln2_b": 7, "w_fc1": 8, "b_fc1": 9, "w_fc2": 10, "b_fc2": 11}


class bf_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("S_hidden", "N_heads", "S_head", "S_mlp", "S_seq", "N_layers", "N_mb_max",
                                         "S_mb_max", "dtype", "ckpt_mode", "causal", "kernels", "queue_depth",
                                         "fuse_wgrad", "N_loop_min", "dp_fs", "S_voc")] + \
               [("seed", C.c_uint64)] + \
               [(n, C.c_float) for n in ("init_std", "ln_eps", "lr", "beta1", "beta2", "adam_eps", "weight_decay")] + \
               [("mb_chains", C.c_int32)]


class bf_event(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("op", "stage", "mb", "live_ckpt")]


class bf_step_report(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("gpu_ms", "adam_ms", "flops_model", "flops_paper", "flops_executed")] + \
               [(n, C.c_int64) for n in ("peak_ckpt_count", "peak_ckpt_bytes", "peak_act_bytes", "state_bytes")] + \
               [("n_events", C.c_int32), ("timed", C.c_int32)] + \
               [("kernel_ms", C.c_double * 11), ("kernel_flops", C.c_double * 11), ("kernel_bytes", C.c_double * 11),
                ("kernel_launches", C.c_int64 * 11)] + \
               [(n, C.c_int64) for n in ("n_weight_intervals", "n_reconstruct", "reconstruct_bytes", "weight_buffer_bytes",
                                         "fused_wgrad_bytes", "mb_chains")]


KERNEL_CLASSES = ("gemm_fwd", "gemm_dgrad", "gemm_wgrad", "attn_fwd", "attn_bwd", "ln_fwd", "ln_bwd", "colsum", "adam",
                  "reconstruct", "vocab")


BF_METHOD_NO_PIPELINE, BF_METHOD_NON_LOOPED, BF_METHOD_DEPTH_FIRST, BF_METHOD_BREADTH_FIRST = range(4)


class bf_calc_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("method", "N_PP", "N_loop", "N_TP", "N_layers", "N_mb", "S_mb", "sharded",
                                         "overlap")] + [("beta_net", C.c_double)]


class bf_calc_point(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("beta", "bubble", "net_ratio", "overlap_share", "net_overhead", "efficiency")]


class bf_sched_stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("makespan", "busy", "bubble_num", "bubble_den", "peak_live")]


class bf_attn_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "kernels", "S_mb", "S_seq", "N_heads", "N_kv_heads", "S_head")] + \
               [("scale", C.c_float), ("cap", C.c_float)] + [(n, C.c_int64) for n in ("ld_q", "ld_k", "ld_v", "ld_ctx")]


class bf_adam_tensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w", "m", "v", "g", "w_lp")] + [("n", C.c_size_t)]


_P = C.c_void_p
_FP = C.POINTER(C.c_float)
_SIGNATURES = {
    "bf_workspace_bytes": (C.c_size_t, [C.POINTER(bf_config)]),
    "bf_create_stack": (C.c_int, [C.POINTER(bf_config), _P, C.c_size_t, _P, C.POINTER(_P)]),
    "bf_destroy_stack": (C.c_int, [_P]),
    "bf_tensor_elems": (C.c_size_t, [_P, C.c_int]),
    "bf_set_params": (C.c_int, [_P, C.c_int, C.c_int, _P, C.c_size_t]),
    "bf_get_params": (C.c_int, [_P, C.c_int, C.c_int, _P, C.c_size_t]),
    "bf_get_grads": (C.c_int, [_P, C.c_int, C.c_int, _P, C.c_size_t]),
    "bf_get_moments": (C.c_int, [_P, C.c_int, C.c_int, C.c_int, _P, C.c_size_t]),
    "bf_reset_optimizer": (C.c_int, [_P]),
    "bf_run_step": (C.c_int, [_P, C.c_int, C.c_int, C.c_int, C.c_int, _P, _P, _P, _P, C.c_int, C.c_int, _P,
                              C.POINTER(bf_step_report)]),
    "bf_run_lm_step": (C.c_int, [_P, C.c_int, C.c_int, C.c_int, C.c_int, _P, _P, _P, C.c_int, C.c_int, _P,
                                 C.POINTER(bf_step_report)]),
    "bf_run_rank_step": (C.c_int, [_P, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, _P, _P, _P, _P, C.c_int, C.c_int, _P,
                              C.POINTER(bf_step_report)]),
    "bf_get_launch_counts": (C.c_int, [_P, C.POINTER(C.c_int64)]),
    "bf_get_trace": (C.c_int, [_P, C.POINTER(bf_event), C.c_size_t, C.POINTER(C.c_size_t)]),
    "bf_schedule_trace": (C.c_int, [C.c_int] * 7 + [C.POINTER(bf_event), C.c_size_t, C.POINTER(C.c_size_t),
                                                    C.POINTER(bf_sched_stats)]),
    "bf_param_count": (C.c_int64, [C.POINTER(bf_config)]),
    "bf_calc_efficiency": (C.c_int, [C.POINTER(bf_calc_config), C.POINTER(bf_calc_point)]),
    "bf_calc_efficiency_curve": (C.c_int, [C.POINTER(bf_calc_config), C.POINTER(C.c_int32), C.c_size_t,
                                           C.POINTER(bf_calc_point)]),
    "bf_calc_beta_threshold": (C.c_int, [C.POINTER(bf_calc_config), C.POINTER(C.c_double)]),
    "bf_calc_cost_time": (C.c_int, [C.c_double] * 4 + [C.POINTER(C.c_double)] * 2),
    "bf_last_error": (C.c_char_p, []),
    "bf_op_gemm": (C.c_int, [C.c_int] * 7 + [_P] * 6 + [C.c_int, _P]),
    "bf_op_gemm_gelu_bwd_colsum": (C.c_int, [C.c_int] * 5 + [_P] * 6 + [C.c_int, _P]),
    "bf_op_gemm_uses_mfma": (C.c_int, [C.c_int] * 5),
    "bf_op_gemm_tile": (C.c_int, [C.c_int] * 5 + [C.POINTER(C.c_int)] * 2),
    "bf_op_wgrad": (C.c_int, [C.c_int] * 6 + [_P, C.c_size_t, _P, C.c_size_t, _P, _P, C.c_int, _P]),
    "bf_op_layernorm_fwd": (C.c_int, [C.c_int, C.c_int, C.c_int, _P, _P, _P, C.c_float, _P, _P, _P]),
    "bf_op_layernorm_bwd": (C.c_int, [C.c_int, C.c_int, C.c_int] + [_P] * 8 + [C.c_int, _P]),
    "bf_op_layernorm_bwd_fused": (C.c_int, [C.c_int, C.c_int, C.c_int] + [_P] * 10 + [C.c_int, _P]),
    "bf_op_layernorm_bwd_part_elems": (C.c_size_t, [C.c_int, C.c_int]),
    "bf_op_colsum": (C.c_int, [C.c_int, C.c_int, C.c_int, _P, _P, C.c_int, _P]),
    "bf_op_attention_fwd": (C.c_int, [C.c_int] * 7 + [_P] * 4),
    "bf_op_attention_bwd": (C.c_int, [C.c_int] * 7 + [_P] * 7),
    "bf_op_attention_bwd_static": (C.c_int, [C.c_int] * 7 + [_P] * 6),
    "bf_op_gemm_splitk": (C.c_int, [C.c_int] * 7 + [_P] * 6 + [C.c_size_t, _P]),
    "bf_op_gemm_splitk_slices": (C.c_int, [C.c_int] * 5),
    "bf_op_attention_bwd_bias": (C.c_int, [C.c_int] * 7 + [_P] * 8 + [C.c_int, _P]),
    "bf_op_attention_bwd_part_elems": (C.c_size_t, [C.c_int] * 4),
    "bf_op_attention_uses_mfma": (C.c_int, [C.c_int, C.c_int]),
    "bf_op_embedding_fwd": (C.c_int, [C.c_int] * 5 + [_P, _P, _P, _P, _P]),
    "bf_op_embedding_bwd": (C.c_int, [C.c_int] * 5 + [_P, _P, _P, _P, C.c_int, _P]),
    "bf_op_ce_loss": (C.c_int, [C.c_int] * 3 + [_P, _P, C.c_float, _P, _P, _P]),
    "bf_op_attention_spans_elems": (C.c_size_t, [C.c_int] * 2),
    "bf_op_attention_spans": (C.c_int, [C.c_int] * 3 + [_P] * 4),
    "bf_op_attention_masked_fwd": (C.c_int, [_P] * 9),
    "bf_op_attention_masked_bwd_work_bytes": (C.c_size_t, [_P]),
    "bf_op_attention_masked_bwd": (C.c_int, [_P] * 13 + [C.c_size_t, _P]),
    "bf_op_vocab_loss_work_bytes": (C.c_size_t, [C.c_int] * 6),
    "bf_op_vocab_loss_fwd": (C.c_int, [C.c_int] * 5 + [_P, _P, _P, C.c_float, _P, _P, _P, _P, C.c_size_t, _P]),
    "bf_op_vocab_loss_bwd": (C.c_int, [C.c_int] * 5 + [_P, _P, _P, _P, C.c_float, _P, _P, C.c_int, _P, C.c_size_t, _P]),
    "bf_op_grad_norm_work_bytes": (C.c_size_t, [C.c_int, _P]),
    "bf_op_grad_norm": (C.c_int, [C.c_int, C.c_int, _P, _P, C.c_float, _P, _P, C.c_size_t, _P]),
    "bf_op_grad_scale": (C.c_int, [C.c_int, C.c_int, _P, _P, _P, _P, _P]),
    "bf_op_adam_clipped": (C.c_int, [C.c_int, _P, _P, C.c_int] + [C.c_float] * 5 + [_P]),
    "bf_op_adam": (C.c_int, [C.c_size_t, _P, _P, _P, _P, _P, C.c_int] + [C.c_float] * 5 + [_P]),
}

_lib = None


class BfError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("libbf status %d: %s" % (status, text))
        self.status = status


def load():
    """Loads libbf.so (built by paper_2211_05953_amd.build); raises ImportError if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libbf.so is not built: run `python -m paper_2211_05953_amd.build`")
        lib = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def last_error():
    return load().bf_last_error().decode()


def check(status):
    if status != BF_OK:
        raise BfError(status, last_error())


def _ptr(t):
    """Device (or host) address of a torch tensor / numpy array / None."""
    if t is None:
        return None
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


def _stream():
    """Handle of the current stream of the current device, without building a torch stream object around it (2.9 -> 0.2 us
    of a call that takes 4 to 6: small kernels are bound by the host)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def make_config(S_hidden, N_heads, S_mlp, S_seq, N_layers, N_mb_max, S_mb_max, dtype=BF_BF16, ckpt_mode=BF_CKPT_NONE,
                causal=1, kernels=BF_KERNELS_AUTO, queue_depth=0, fuse_wgrad=0, N_loop_min=0, dp_fs=0, S_voc=0, seed=0x221105953, init_std=0.02, ln_eps=1e-5,
                lr=1e-4, beta1=0.9, beta2=0.999, adam_eps=1e-8, weight_decay=0.0, mb_chains=1):
    return bf_config(S_hidden, N_heads, S_hidden // N_heads, S_mlp, S_seq, N_layers, N_mb_max, S_mb_max, dtype,
                     ckpt_mode, causal, kernels, queue_depth, fuse_wgrad, N_loop_min, dp_fs, S_voc, seed, init_std, ln_eps, lr, beta1, beta2, adam_eps,
                     weight_decay, mb_chains)


def bf_workspace_bytes(cfg):
    return load().bf_workspace_bytes(C.byref(cfg))


def bf_param_count(cfg):
    return load().bf_param_count(C.byref(cfg))


class Stack:
    """Owns the torch-allocated workspace and the opaque bf_stack handle."""

    def __init__(self, cfg, device="cuda:0"):
        import torch
        lib = load()
        self.cfg = cfg
        n = lib.bf_workspace_bytes(C.byref(cfg))
        if n == 0:
            raise BfError(BF_EINVAL, last_error())
        self.workspace = torch.empty(n, dtype=torch.uint8, device=device)
        self.handle = _P()
        with torch.cuda.device(self.workspace.device):
            check(lib.bf_create_stack(C.byref(cfg), self.workspace.data_ptr(), n, _stream(), C.byref(self.handle)))
        self.torch_dtype = torch.bfloat16 if cfg.dtype == BF_BF16 else torch.float32

    def close(self):
        if self.handle:
            load().bf_destroy_stack(self.handle)
            self.handle = _P()
            self.workspace = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def bf_tensor_elems(self, tensor_id):
        return load().bf_tensor_elems(self.handle, tensor_id)

    def _xfer(self, fn, layer, tensor_id, arr, *extra):
        import numpy as np
        assert arr.dtype == np.float32 and arr.flags["C_CONTIGUOUS"]
        check(fn(self.handle, layer, tensor_id, *extra, arr.ctypes.data, arr.size))

    def bf_set_params(self, layer, tensor_id, host_src):
        import numpy as np
        self._xfer(load().bf_set_params, layer, tensor_id, np.ascontiguousarray(host_src, dtype=np.float32))

    def _get(self, fn, layer, tensor_id, *extra):
        import numpy as np
        out = np.empty(self.bf_tensor_elems(tensor_id), dtype=np.float32)
        self._xfer(fn, layer, tensor_id, out, *extra)
        return out

    def bf_get_params(self, layer, tensor_id):
        return self._get(load().bf_get_params, layer, tensor_id)

    def bf_get_grads(self, layer, tensor_id):
        return self._get(load().bf_get_grads, layer, tensor_id)

    def bf_get_moments(self, layer, tensor_id, which):
        return self._get(load().bf_get_moments, layer, tensor_id, which)

    def bf_reset_optimizer(self):
        check(load().bf_reset_optimizer(self.handle))

    def bf_run_step(self, schedule, N_loop, N_mb, S_mb, x, dy, y=None, dx=None, apply_optimizer=0, timing=0):
        rep = bf_step_report()
        check(load().bf_run_step(self.handle, schedule, N_loop, N_mb, S_mb, _ptr(x), _ptr(dy), _ptr(y), _ptr(dx),
                                 apply_optimizer, timing, _stream(), C.byref(rep)))
        return rep

    def bf_run_lm_step(self, schedule, N_loop, N_mb, S_mb, tokens, labels, loss, apply_optimizer=0, timing=0):
        rep = bf_step_report()
        check(load().bf_run_lm_step(self.handle, schedule, N_loop, N_mb, S_mb, _ptr(tokens), _ptr(labels), _ptr(loss),
                                    apply_optimizer, timing, _stream(), C.byref(rep)))
        return rep

    def bf_run_rank_step(self, schedule, N_PP, rank, N_loop, N_mb, S_mb, x, dy, y=None, dx=None, apply_optimizer=0,
                         timing=0):
        rep = bf_step_report()
        check(load().bf_run_rank_step(self.handle, schedule, N_PP, rank, N_loop, N_mb, S_mb, _ptr(x), _ptr(dy), _ptr(y),
                                      _ptr(dx), apply_optimizer, timing, _stream(), C.byref(rep)))
        return rep

    def bf_get_trace(self):
        n = C.c_size_t(0)
        check(load().bf_get_trace(self.handle, None, 0, C.byref(n)))
        buf = (bf_event * max(1, n.value))()
        check(load().bf_get_trace(self.handle, buf, n.value, C.byref(n)))
        return [(e.op, e.stage, e.mb, e.live_ckpt) for e in buf[:n.value]]

    def bf_get_launch_counts(self):
        """Timed launches of the last step as made, in the order of KERNEL_CLASSES."""
        buf = (C.c_int64 * len(KERNEL_CLASSES))()
        check(load().bf_get_launch_counts(self.handle, buf))
        return list(buf)


def bf_schedule_trace(schedule, N_PP, N_loop, N_mb, rank, t_fwd=1, t_bwd=2):
    """Returns (events, stats) of the pure-host schedule generator."""
    lib = load()
    n = C.c_size_t(0)
    check(lib.bf_schedule_trace(schedule, N_PP, N_loop, N_mb, rank, t_fwd, t_bwd, None, 0, C.byref(n), None))
    buf = (bf_event * max(1, n.value))()
    st = bf_sched_stats()
    check(lib.bf_schedule_trace(schedule, N_PP, N_loop, N_mb, rank, t_fwd, t_bwd, buf, n.value, C.byref(n), C.byref(st)))
    return [(e.op, e.stage, e.mb, e.live_ckpt) for e in buf[:n.value]], st


# ---- analytical calculators (include/bf_calc.h); host arithmetic only ------------------------
def _point(p):
    return {n: getattr(p, n) for n, _ in bf_calc_point._fields_}


def bf_calc_efficiency(method, N_PP, N_loop, N_TP, N_layers, N_mb, S_mb, sharded, overlap, beta_net):
    cfg = bf_calc_config(method, N_PP, N_loop, N_TP, N_layers, N_mb, S_mb, sharded, overlap, beta_net)
    out = bf_calc_point()
    check(load().bf_calc_efficiency(C.byref(cfg), C.byref(out)))
    return _point(out)


def bf_calc_efficiency_curve(method, N_PP, N_loop, N_TP, N_layers, S_mb, sharded, overlap, beta_net, n_mb):
    cfg = bf_calc_config(method, N_PP, N_loop, N_TP, N_layers, 1, S_mb, sharded, overlap, beta_net)
    counts = (C.c_int32 * len(n_mb))(*n_mb)
    out = (bf_calc_point * max(1, len(n_mb)))()
    check(load().bf_calc_efficiency_curve(C.byref(cfg), counts, len(n_mb), out))
    return [_point(p) for p in out[:len(n_mb)]]


def bf_calc_beta_threshold(method, N_PP, N_loop, N_TP, N_layers, N_mb, S_mb, sharded, overlap, beta_net):
    cfg = bf_calc_config(method, N_PP, N_loop, N_TP, N_layers, N_mb, S_mb, sharded, overlap, beta_net)
    out = C.c_double(0.0)
    check(load().bf_calc_beta_threshold(C.byref(cfg), C.byref(out)))
    return out.value


def bf_calc_cost_time(beta, N_gpu, B_crit, efficiency=1.0):
    cost, time = C.c_double(0.0), C.c_double(0.0)
    check(load().bf_calc_cost_time(beta, N_gpu, B_crit, efficiency, C.byref(cost), C.byref(time)))
    return cost.value, time.value


# ---- single kernels (include/bf_ops.h); tensors are torch CUDA tensors ----------------------
def bf_op_gemm(dtype, kernels, layout, epilogue, M, N, K, A, B, Cout, bias=None, R=None, C2=None, accumulate=0):
    check(load().bf_op_gemm(dtype, kernels, layout, epilogue, M, N, K, _ptr(A), _ptr(B), _ptr(Cout), _ptr(bias), _ptr(R),
                            _ptr(C2), accumulate, _stream()))


def bf_op_wgrad(dtype, kernels, M, N, K, n_seg, X, stride_x, dY, stride_dy, G, db=None, accumulate=0):
    check(load().bf_op_wgrad(dtype, kernels, M, N, K, n_seg, _ptr(X), stride_x, _ptr(dY), stride_dy, _ptr(G), _ptr(db),
                             accumulate, _stream()))


def bf_op_gemm_gelu_bwd_colsum(dtype, kernels, M, N, K, A, Bt, Cout, R, db, part=None, accumulate=0):
    check(load().bf_op_gemm_gelu_bwd_colsum(dtype, kernels, M, N, K, _ptr(A), _ptr(Bt), _ptr(Cout), _ptr(R), _ptr(db),
                                            _ptr(part), accumulate, _stream()))


def bf_op_gemm_splitk(dtype, kernels, layout, epilogue, M, N, K, A, B, Cout, bias=None, R=None, planes=None):
    opt = lambda t: _ptr(t) if t is not None else None
    check(load().bf_op_gemm_splitk(dtype, kernels, layout, epilogue, M, N, K, _ptr(A), _ptr(B), _ptr(Cout), opt(bias), opt(R),
                                   opt(planes), planes.numel() if planes is not None else 0, _stream()))


def bf_op_gemm_splitk_slices(layout, epilogue, M, N, K):
    return load().bf_op_gemm_splitk_slices(layout, epilogue, M, N, K)


def bf_op_gemm_uses_mfma(layout, epilogue, M, N, K):
    return bool(load().bf_op_gemm_uses_mfma(layout, epilogue, M, N, K))


def bf_op_gemm_tile(layout, epilogue, M, N, K):
    """(rows, columns) of the MFMA kernel's tile for this product, or None where the plain kernel runs."""
    bm, bn = C.c_int(0), C.c_int(0)
    ok = load().bf_op_gemm_tile(layout, epilogue, M, N, K, C.byref(bm), C.byref(bn))
    return (bm.value, bn.value) if ok else None


def bf_op_layernorm_fwd(dtype, T, h, x, g, b, eps, y, stats):
    check(load().bf_op_layernorm_fwd(dtype, T, h, _ptr(x), _ptr(g), _ptr(b), eps, _ptr(y), _ptr(stats), _stream()))


def bf_op_layernorm_bwd(dtype, T, h, dy, x, g, stats, dres, dx, dg, db, accumulate=0):
    check(load().bf_op_layernorm_bwd(dtype, T, h, _ptr(dy), _ptr(x), _ptr(g), _ptr(stats), _ptr(dres), _ptr(dx),
                                     _ptr(dg), _ptr(db), accumulate, _stream()))


def bf_op_layernorm_bwd_fused(dtype, T, h, dy, x, g, stats, dres, dx, dg, db, dcs=None, part=None, accumulate=0):
    check(load().bf_op_layernorm_bwd_fused(dtype, T, h, _ptr(dy), _ptr(x), _ptr(g), _ptr(stats), _ptr(dres), _ptr(dx),
                                           _ptr(dg), _ptr(db), _ptr(dcs), _ptr(part), accumulate, _stream()))


def bf_op_layernorm_bwd_part_elems(T, h):
    return load().bf_op_layernorm_bwd_part_elems(T, h)


def bf_op_colsum(dtype, T, N, dY, out, accumulate=0):
    check(load().bf_op_colsum(dtype, T, N, _ptr(dY), _ptr(out), accumulate, _stream()))


def bf_op_attention_fwd(dtype, kernels, S_mb, S_seq, N_heads, S_head, causal, qkv, ctx, lse):
    check(load().bf_op_attention_fwd(dtype, kernels, S_mb, S_seq, N_heads, S_head, causal, _ptr(qkv), _ptr(ctx),
                                     _ptr(lse), _stream()))


def bf_op_attention_bwd(dtype, kernels, S_mb, S_seq, N_heads, S_head, causal, qkv, ctx, lse, dctx, dqkv, delta):
    check(load().bf_op_attention_bwd(dtype, kernels, S_mb, S_seq, N_heads, S_head, causal, _ptr(qkv), _ptr(ctx),
                                     _ptr(lse), _ptr(dctx), _ptr(dqkv), _ptr(delta), _stream()))


def bf_op_attention_bwd_bias(dtype, kernels, S_mb, S_seq, N_heads, S_head, causal, qkv, ctx, lse, dctx, dqkv, delta, db_qkv,
                             part=None, accumulate=0):
    check(load().bf_op_attention_bwd_bias(dtype, kernels, S_mb, S_seq, N_heads, S_head, causal, _ptr(qkv), _ptr(ctx),
                                          _ptr(lse), _ptr(dctx), _ptr(dqkv), _ptr(delta), _ptr(db_qkv),
                                          _ptr(part) if part is not None else None, int(accumulate), _stream()))


def bf_op_attention_bwd_part_elems(S_mb, S_seq, N_heads, S_head):
    return load().bf_op_attention_bwd_part_elems(S_mb, S_seq, N_heads, S_head)


def bf_op_attention_bwd_static(dtype, kernels, S_mb, S_seq, N_heads, S_head, causal, qkv, ctx, lse, dctx, dqkv):
    check(load().bf_op_attention_bwd_static(dtype, kernels, S_mb, S_seq, N_heads, S_head, causal, _ptr(qkv), _ptr(ctx),
                                            _ptr(lse), _ptr(dctx), _ptr(dqkv), _stream()))


def bf_op_attention_uses_mfma(S_seq, S_head):
    return bool(load().bf_op_attention_uses_mfma(S_seq, S_head))


def bf_op_embedding_fwd(dtype, n_rows, S_seq, S_voc, S_hidden, tokens, e_tok, e_pos, x):
    check(load().bf_op_embedding_fwd(dtype, n_rows, S_seq, S_voc, S_hidden, _ptr(tokens), _ptr(e_tok), _ptr(e_pos), _ptr(x),
                                     _stream()))


def bf_op_embedding_bwd(dtype, S_mb, S_seq, S_voc, S_hidden, tokens, d, g_tok, g_pos, accumulate_pos):
    check(load().bf_op_embedding_bwd(dtype, S_mb, S_seq, S_voc, S_hidden, _ptr(tokens), _ptr(d), _ptr(g_tok), _ptr(g_pos),
                                     accumulate_pos, _stream()))


def bf_op_ce_loss(dtype, n_rows, S_voc, z, labels, scale, row_loss, loss_out):
    check(load().bf_op_ce_loss(dtype, n_rows, S_voc, _ptr(z), _ptr(labels), scale, _ptr(row_loss), _ptr(loss_out), _stream()))


def bf_op_adam(n, w, m, v, g, w_lp, t, lr, beta1, beta2, adam_eps, weight_decay):
    check(load().bf_op_adam(n, _ptr(w), _ptr(m), _ptr(v), _ptr(g), _ptr(w_lp), t, lr, beta1, beta2, adam_eps,
                            weight_decay, _stream()))


_torch = None


def _th():
    """torch, imported on first use: the calculators and the schedule need none of it."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _torch_dtype(dtype):
    return _th().bfloat16 if dtype == BF_BF16 else _th().float32


def _tensors(who, tensors, dtype):
    """Checks tensors that a kernel is to work on: dense, of `dtype` (torch), on the current device."""
    dev = _th()._C._cuda_getDevice()
    for t in tensors:
        if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
            raise ValueError("%s: needs contiguous %s tensors on cuda:%d, got %s on %s, strides %s" % (who, dtype, dev, t.dtype, t.device, t.stride()))


def _elems(who, tensor, n):
    if tensor.numel() < n:
        raise ValueError("%s: a tensor of %d elements where %d are used" % (who, tensor.numel(), n))


def _work(who, work, n):
    """The caller's scratch, or n bytes from torch's allocator (in the current stream's order)."""
    if work is None:
        return _th().empty(n or 1, dtype=_th().uint8, device="cuda")
    _tensors(who, (work,), work.dtype)
    return work


def _list(who, tensors, dtype):
    """Host arrays of the addresses and sizes of a list of tensors, checked as by _tensors.  (Hundreds of tensors: the checks
    of one kind together, a few calls into torch each.)"""
    if [t.dtype for t in tensors].count(dtype) != len(tensors) or \
            [t.get_device() for t in tensors].count(_th()._C._cuda_getDevice()) != len(tensors) or not all([t.is_contiguous() for t in tensors]):
        _tensors(who, tensors, dtype)
    return _array("Q", [t.data_ptr() for t in tensors]), _array("Q", [t.numel() for t in tensors])


def _at(arr):
    """Address of an array's elements, NULL for an empty one.  The array itself has to live until the call is over."""
    return arr.buffer_info()[0] if len(arr) else None


def make_attn_config(dtype, S_mb, S_seq, N_heads, N_kv_heads, S_head, scale=0.0, cap=0.0, ld_q=0, ld_k=0, ld_v=0, ld_ctx=0, kernels=BF_KERNELS_AUTO):
    return bf_attn_config(dtype, kernels, S_mb, S_seq, N_heads, N_kv_heads, S_head, scale, cap, ld_q, ld_k, ld_v, ld_ctx)


def bf_op_attention_spans_elems(S_mb, S_seq):
    return load().bf_op_attention_spans_elems(S_mb, S_seq)


def bf_op_attention_spans(S_mb, S_seq, causal, doc, prefix, spans):
    """spans (int32, bf_op_attention_spans_elems) from document ids [S_mb, S_seq] and prefix lengths [S_mb], int32 or None each."""
    who = "bf_op_attention_spans"
    _tensors(who, [t for t in (doc, prefix, spans) if t is not None], _th().int32)
    for t, n in ((doc, S_mb * S_seq), (prefix, S_mb), (spans, bf_op_attention_spans_elems(S_mb, S_seq))):
        if t is not None:
            _elems(who, t, n)
    check(load().bf_op_attention_spans(S_mb, S_seq, causal, _ptr(doc), _ptr(prefix), _ptr(spans), _stream()))


def _token_rows(t, S_mb, S_seq, heads, S_head, ld):
    """Whether token (b, s) of `t` starts where the kernels look for it, (b S_seq + s) ld elements in, its heads side by side.  The dimensions are
    (sequences, tokens, row) or (all tokens, row), the row one or several that end in S_head, or one for everything; there may be more
    sequences, tokens or columns than are used."""
    n = heads * S_head
    step = ld or n
    shape, stride = t.shape, t.stride()
    for lead in (((S_mb, S_seq * step), (S_seq, step)), ((S_mb * S_seq, step),)):
        at = len(lead)
        if t.dim() <= at or (t.dim() > at + 1 and shape[-1] != S_head):
            continue
        dense = 1  # elements of the row's inner dimensions; a step is met by nothing if one is used
        fits = all(size >= used and (used == 1 or x == want) for size, x, (used, want) in zip(shape, stride, lead))
        for size, x in zip(reversed(shape[at:]), reversed(stride[at:])):
            fits = fits and (size == 1 or x == dense)
            dense *= size
        if fits and dense >= n:
            return True
    return t.dim() == 1 and shape[0] >= (S_mb * S_seq - 1) * step + n and (shape[0] == 1 or stride[0] == 1)


def _attn_tensors(who, cfg, spans, slopes, lse, rows):
    """rows: (tensor, heads, step from a token to the next) each; the tensors may be views into longer rows."""
    torch = _th()
    dev, dtype = torch._C._cuda_getDevice(), _torch_dtype(cfg.dtype)
    S_mb, S_seq, S_head = cfg.S_mb, cfg.S_seq, cfg.S_head
    for t, heads, ld in rows:
        n = heads * S_head
        if t.dtype is not dtype or t.get_device() != dev:
            raise ValueError("%s: needs %s tensors on cuda:%d, got %s on %s" % (who, dtype, dev, t.dtype, t.device))
        if t.dim() == 3 and t.shape == (S_mb, S_seq, n) and t.stride() == (S_seq * (ld or n), ld or n, 1):
            continue
        if not _token_rows(t, S_mb, S_seq, heads, S_head, ld):
            raise ValueError("%s: a tensor of shape %s and strides %s is not %d x %d tokens of %d heads of %d, %d elements apart"
                             % (who, tuple(t.shape), t.stride(), S_mb, S_seq, heads, S_head, ld or n))
    _tensors(who, (spans,), torch.int32)
    _elems(who, spans, bf_op_attention_spans_elems(S_mb, S_seq))
    if slopes is not None:
        _tensors(who, (slopes,), torch.float32)
        _elems(who, slopes, cfg.N_heads)
    if lse is not None:
        _tensors(who, (lse,), torch.float32)
        _elems(who, lse, S_mb * cfg.N_heads * S_seq)


def bf_op_attention_masked_fwd(cfg, q, k, v, spans, slopes, ctx, lse=None):
    _attn_tensors("bf_op_attention_masked_fwd", cfg, spans, slopes, lse,
                  ((q, cfg.N_heads, cfg.ld_q), (k, cfg.N_kv_heads, cfg.ld_k), (v, cfg.N_kv_heads, cfg.ld_v), (ctx, cfg.N_heads, cfg.ld_ctx)))
    check(load().bf_op_attention_masked_fwd(C.byref(cfg), q.data_ptr(), k.data_ptr(), v.data_ptr(), spans.data_ptr(), _ptr(slopes), ctx.data_ptr(), _ptr(lse),
                                            _stream()))


def bf_op_attention_masked_bwd_work_bytes(cfg):
    return load().bf_op_attention_masked_bwd_work_bytes(C.byref(cfg))


def bf_op_attention_masked_bwd(cfg, q, k, v, spans, slopes, ctx, lse, dctx, dq, dk, dv, work=None):
    who, h, kv = "bf_op_attention_masked_bwd", cfg.N_heads, cfg.N_kv_heads
    _attn_tensors(who, cfg, spans, slopes, lse, ((q, h, cfg.ld_q), (k, kv, cfg.ld_k), (v, kv, cfg.ld_v), (ctx, h, cfg.ld_ctx), (dctx, h, cfg.ld_ctx),
                                                 (dq, h, cfg.ld_q), (dk, kv, cfg.ld_k), (dv, kv, cfg.ld_v)))
    work = _work(who, work, bf_op_attention_masked_bwd_work_bytes(cfg))
    check(load().bf_op_attention_masked_bwd(C.byref(cfg), q.data_ptr(), k.data_ptr(), v.data_ptr(), spans.data_ptr(), _ptr(slopes), ctx.data_ptr(),
                                            lse.data_ptr(), dctx.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), work.data_ptr(),
                                            work.numel() * work.element_size(), _stream()))


def bf_op_vocab_loss_work_bytes(dtype, n_rows, S_hidden, S_voc, S_piece=0, backward=0):
    return load().bf_op_vocab_loss_work_bytes(dtype, n_rows, S_hidden, S_voc, S_piece, backward)


def _vocab_loss(who, dtype, n_rows, S_hidden, S_voc, S_piece, backward, y, w_out, labels, fp32, small, work):
    torch = _th()
    _tensors(who, (y, w_out), _torch_dtype(dtype))
    _tensors(who, (labels,), torch.int32)
    _tensors(who, fp32, torch.float32)
    _elems(who, y, n_rows * S_hidden)
    _elems(who, w_out, S_voc * S_hidden)
    for t in (labels,) + small:
        _elems(who, t, n_rows)
    return _work(who, work, load().bf_op_vocab_loss_work_bytes(dtype, n_rows, S_hidden, S_voc, S_piece, backward))


def bf_op_vocab_loss_fwd(dtype, n_rows, S_hidden, S_voc, y, w_out, labels, scale, lse, row_loss, loss_out, S_piece=0, work=None):
    who = "bf_op_vocab_loss_fwd"
    work = _vocab_loss(who, dtype, n_rows, S_hidden, S_voc, S_piece, 0, y, w_out, labels, (lse, row_loss, loss_out), (lse, row_loss), work)
    _elems(who, loss_out, 1)
    check(load().bf_op_vocab_loss_fwd(dtype, n_rows, S_hidden, S_voc, S_piece, y.data_ptr(), w_out.data_ptr(), labels.data_ptr(), scale, lse.data_ptr(),
                                      row_loss.data_ptr(), loss_out.data_ptr(), work.data_ptr(), work.numel() * work.element_size(), _stream()))


def bf_op_vocab_loss_bwd(dtype, n_rows, S_hidden, S_voc, y, w_out, labels, lse, scale, dy, dw, accumulate=0, S_piece=0, work=None):
    who = "bf_op_vocab_loss_bwd"
    work = _vocab_loss(who, dtype, n_rows, S_hidden, S_voc, S_piece, 1, y, w_out, labels, (lse, dw), (lse,), work)
    _tensors(who, (dy,), _torch_dtype(dtype))
    _elems(who, dy, n_rows * S_hidden)
    _elems(who, dw, S_voc * S_hidden)
    check(load().bf_op_vocab_loss_bwd(dtype, n_rows, S_hidden, S_voc, S_piece, y.data_ptr(), w_out.data_ptr(), labels.data_ptr(), lse.data_ptr(), scale,
                                      dy.data_ptr(), dw.data_ptr(), accumulate, work.data_ptr(), work.numel() * work.element_size(), _stream()))


def bf_op_grad_norm_work_bytes(tensors):
    n = _array("Q", [t.numel() for t in tensors])
    return load().bf_op_grad_norm_work_bytes(len(n), _at(n))


def bf_op_grad_norm(dtype, tensors, max_norm, out, work=None):
    """out (fp32, 2 elements) = norm over a list of gradients, coefficient that clips it to max_norm."""
    who = "bf_op_grad_norm"
    lib, (g, n) = load(), _list(who, tensors, _torch_dtype(dtype))
    _tensors(who, (out,), _th().float32)
    _elems(who, out, 2)
    work = _work(who, work, lib.bf_op_grad_norm_work_bytes(len(g), _at(n)))
    check(lib.bf_op_grad_norm(dtype, len(g), _at(g), _at(n), max_norm, out.data_ptr(), work.data_ptr(), work.numel() * work.element_size(), _stream()))


def bf_op_grad_scale(dtype, tensors, dst, coef):
    """dst[i] = tensors[i] * coef (device fp32); dst may be the tensors themselves."""
    who = "bf_op_grad_scale"
    (g, n), (d, m) = _list(who, tensors, _torch_dtype(dtype)), _list(who, dst, _torch_dtype(dtype))
    _tensors(who, (coef,), _th().float32)
    _elems(who, coef, 1)
    if n != m:
        raise ValueError("%s: the lists differ in their sizes" % who)
    check(load().bf_op_grad_scale(dtype, len(g), _at(g), _at(d), _at(n), coef.data_ptr(), _stream()))


def bf_op_adam_clipped(tensors, coef, t, lr, beta1, beta2, adam_eps, weight_decay):
    """The Adam step number t on gradients times coef (device fp32).  tensors: (w, m, v, g, w_lp) each, w_lp bf16 or None."""
    who, torch = "bf_op_adam_clipped", _th()
    _tensors(who, (coef,), torch.float32)
    _elems(who, coef, 1)
    w, m, v, g, low = zip(*tensors) if tensors else ((),) * 5
    (pw, n), (pm, n1), (pv, n2), (pg, n3) = (_list(who, x, torch.float32) for x in (w, m, v, g))
    pl, n4 = _list(who, [x for x in low if x is not None], torch.bfloat16)
    if not n == n1 == n2 == n3 or n4 != _array("Q", [k for k, x in zip(n, low) if x is not None]):
        raise ValueError("%s: tensors of different sizes in one entry" % who)
    rest = iter(pl)
    a = _array("Q", [x for i, k in enumerate(n) for x in (pw[i], pm[i], pv[i], pg[i], 0 if low[i] is None else next(rest), k)])  # bf_adam_tensor
    check(load().bf_op_adam_clipped(len(n), _at(a), coef.data_ptr(), t, lr, beta1, beta2, adam_eps, weight_decay, _stream()))
