"""Python binding of libmist (include/mist.h): argument marshalling only.

Every step of the tuner's hot path runs inside libmist.so (host space build and HIP
kernels on the GPU).  PyTorch provides device memory (its caching allocator, through the
library's allocator callbacks) and the stream.  If the library is missing this module
raises; there is no fallback.
"""

from __future__ import annotations

import collections
import ctypes
import math
import os
import threading

import numpy as np

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libmist.so")

MIST_NONE = 0xFFFFFFFFFFFFFFFF
NONE = np.uint64(MIST_NONE)

EXPORTS = [
    "mist_space_create", "mist_eval_space", "mist_get_best", "mist_get_pareto", "mist_get_alpha",
    "mist_get_buckets",
    "mist_space_info", "mist_get_group_key", "mist_decode", "mist_eval_ids", "mist_set_timing",
    "mist_read_timing", "mist_launch_info", "mist_space_destroy", "mist_last_error",
    "mist_plan_points", "mist_plan_pipeline", "mist_eval_pareto_exact", "mist_get_pareto_exact", "mist_exact_info",
    "mist_corun_create", "mist_corun_run", "mist_corun_reduce", "mist_corun_measure", "mist_corun_destroy",
    "mist_fit_phi", "mist_interference", "mist_measure_eta", "mist_probe_fp64",
    "mist_search_info", "mist_tile_info", "mist_debug_eval_tiles", "mist_eval_ids_noalloc", "mist_exact_group_sizes",
    "mist_embed_forward", "mist_embed_workspace", "mist_embed_backward", "mist_tensors_create", "mist_tensors_destroy",
    "mist_norm_workspace", "mist_grad_norm", "mist_grad_finish", "mist_grad_clip", "mist_adam_step",
    "mist_token_logprob", "mist_token_part", "mist_token_join", "mist_token_grad", "mist_token_loss",
    "mist_block_forward", "mist_block_workspace", "mist_block_backward", "mist_kept_store", "mist_kept_load",
    "mist_act_forward", "mist_act_backward",
]

PROBE_KINDS = {"add": 0, "mul": 1, "fma": 2, "min": 3, "max": 4, "cmp": 5}


class MistError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("libmist status %d: %s" % (status, msg))
        self.status = status


class ModelDesc(ctypes.Structure):
    _fields_ = [("arch", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("hidden", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("ffn", ctypes.c_int64),
                ("seq", ctypes.c_int64), ("vocab", ctypes.c_int64), ("bytes_w", ctypes.c_int32),
                ("bytes_opt", ctypes.c_int32), ("flash", ctypes.c_int32)]


class HwDesc(ctypes.Structure):
    _fields_ = [("flops", ctypes.c_double), ("mem_bytes", ctypes.c_double), ("pcie_bw", ctypes.c_double),
                ("link_bw", ctypes.c_double), ("eta_max", ctypes.c_double), ("n_half", ctypes.c_double),
                ("phi", (ctypes.c_double * 4) * 16), ("eta_tab", ctypes.c_double * 16)]


class SpaceDesc(ctypes.Structure):
    _fields_ = [("n_devices", ctypes.c_int64), ("global_batch", ctypes.c_int64),
                ("mb", ctypes.POINTER(ctypes.c_int32)), ("n_mb", ctypes.c_int32),
                ("ratios", ctypes.POINTER(ctypes.c_double)), ("n_ratios", ctypes.c_int32),
                ("n_buckets", ctypes.c_int32), ("l_rule", ctypes.c_int32),
                ("n_alphas", ctypes.c_int32), ("alphas", ctypes.POINTER(ctypes.c_double)),
                ("tile_configs", ctypes.c_int64), ("max_blocks", ctypes.c_int32),
                ("cand_window", ctypes.c_int32)]


MAX_STAGES = 64
CORUN_MAX_UNITS = 256
CORUN_SAMPLES_PER_SHAPE = 28


class CorunShape(ctypes.Structure):
    _fields_ = [("gemm_m", ctypes.c_int64), ("gemm_n", ctypes.c_int64), ("gemm_k", ctypes.c_int64),
                ("g2g_bytes", ctypes.c_int64), ("h2d_bytes", ctypes.c_int64), ("d2h_bytes", ctypes.c_int64)]


class CorunSample(ctypes.Structure):
    _fields_ = [("mask", ctypes.c_int32), ("stream", ctypes.c_int32), ("shape", ctypes.c_int32),
                ("units", ctypes.c_int32), ("solo_s", ctypes.c_double), ("corun_s", ctypes.c_double)]


class StagePoint(ctypes.Structure):
    _fields_ = [("G", ctypes.c_int32), ("PP", ctypes.c_int32), ("k", ctypes.c_int32), ("l", ctypes.c_int32),
                ("id", ctypes.c_uint64), ("t", ctypes.c_double), ("d", ctypes.c_double)]


class StagePlan(ctypes.Structure):
    _fields_ = [("l", ctypes.c_int32), ("k", ctypes.c_int32), ("id", ctypes.c_uint64),
                ("t", ctypes.c_double), ("d", ctypes.c_double)]


class Plan(ctypes.Structure):
    _fields_ = [("found", ctypes.c_int32), ("hw", ctypes.c_int32), ("G", ctypes.c_int32), ("PP", ctypes.c_int32),
                ("F", ctypes.c_double), ("stage", StagePlan * MAX_STAGES)]


def _plan_dict(p: Plan) -> dict | None:
    if not p.found:
        return None
    return {"hw": p.hw, "G": p.G, "PP": p.PP, "F": p.F,
            "stages": [_struct_to_dict(p.stage[i]) for i in range(p.PP)]}


ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p)
FREE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p)


class Allocator(ctypes.Structure):
    _fields_ = [("alloc", ALLOC_FN), ("free", FREE_FN), ("ctx", ctypes.c_void_p)]


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ["hw", "G", "PP", "k", "l", "b", "tp", "dp", "zero", "ckpt",
                 "wo_idx", "go_idx", "oo_idx", "ao_idx"]] + \
               [(n, ctypes.c_double) for n in ["wo", "go", "oo", "ao"]]


class Result(ctypes.Structure):
    _fields_ = [("id", ctypes.c_uint64), ("obj", ctypes.c_double), ("t", ctypes.c_double),
                ("d", ctypes.c_double), ("mem", ctypes.c_double), ("bucket", ctypes.c_int32),
                ("pad", ctypes.c_int32), ("cfg", Config)]


class GroupKey(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ["hw", "G", "PP", "k", "l", "n_pairs"]] + \
               [("base", ctypes.c_uint64), ("size", ctypes.c_uint64)]


class EmbedDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in
                ["batch", "seq", "hidden", "rows", "vocab_begin", "ids_stride", "act_batch_stride", "act_stride",
                 "table_stride", "pos_stride"]] + \
               [("ids_bytes", ctypes.c_int32), ("act_type", ctypes.c_int32), ("table_type", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class ClipDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("grad_scale", ctypes.c_float), ("max_norm", ctypes.c_double)]


class AdamDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ["lr", "beta1", "beta2", "eps", "weight_decay"]]


class TokenDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in
                ["batch", "seq", "rows", "vocab_begin", "ids_stride", "logits_batch_stride", "logits_stride",
                 "grad_batch_stride", "grad_stride"]] + \
               [("ids_bytes", ctypes.c_int32), ("type", ctypes.c_int32), ("top", ctypes.c_int32), ("scale", ctypes.c_float)]


class BlockDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in
                ["batch", "seq", "hidden", "x_stride", "block_stride", "y_stride", "h_stride", "gate_stride"]] + \
               [(n, ctypes.c_int32) for n in ["kind", "type", "res_type", "weight_type"]] + \
               [(n, ctypes.c_float) for n in ["eps", "res_scale", "block_scale"]] + [("of_sum", ctypes.c_int32)]


class BlockGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ["dh", "dy", "dx", "dblock", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate"]] + \
               [(n, ctypes.c_int64) for n in ["dh_stride", "dy_stride", "dx_stride", "dblock_stride", "dgate_stride"]] + \
               [("accumulate", ctypes.c_int32)]


class KeptDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ["rows", "width", "stride"]] + [("type", ctypes.c_int32)]


class ActDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ["rows", "width", "up_stride", "gate_stride", "out_stride", "again_stride"]] + \
               [("type", ctypes.c_int32), ("kind", ctypes.c_int32)]


class Kept(ctypes.Structure):
    _fields_ = [("values", ctypes.c_void_p), ("exponents", ctypes.c_void_p)]


_lib = None
_lock = threading.Lock()


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Loads libmist.so (built by paper_2503_19050_amd.build); raises when it is missing."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(path):
            raise MistError(-3, "%s is not built; run paper_2503_19050_amd.build.build()" % path)
        L = ctypes.CDLL(path)
        P = ctypes.POINTER
        st = ctypes.c_int32
        vp = ctypes.c_void_p
        L.mist_space_create.argtypes = [P(ModelDesc), P(HwDesc), ctypes.c_int32, P(SpaceDesc), P(Allocator), P(vp)]
        L.mist_eval_space.argtypes = [vp, vp]
        L.mist_get_best.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, P(Result)]
        L.mist_get_pareto.argtypes = [vp, ctypes.c_int64, P(Result), ctypes.c_int32, P(ctypes.c_int32)]
        L.mist_get_alpha.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, P(Result)]
        L.mist_get_buckets.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, P(ctypes.c_uint64),
                                       P(ctypes.c_double), P(ctypes.c_uint64)]
        L.mist_space_info.argtypes = [vp, P(ctypes.c_uint64), P(ctypes.c_int64), P(ctypes.c_int32)]
        L.mist_get_group_key.argtypes = [vp, ctypes.c_int64, P(GroupKey)]
        L.mist_decode.argtypes = [vp, ctypes.c_uint64, P(Config)]
        L.mist_eval_ids.argtypes = [vp, P(ctypes.c_uint64), ctypes.c_int64, P(ctypes.c_double), vp]
        L.mist_eval_ids_noalloc.argtypes = [vp, P(ctypes.c_uint64), ctypes.c_int64, P(ctypes.c_double), vp]
        L.mist_set_timing.argtypes = [vp, ctypes.c_int32]
        L.mist_read_timing.argtypes = [vp, P(ctypes.c_double), P(ctypes.c_double), P(ctypes.c_int64)]
        L.mist_launch_info.argtypes = [vp, P(ctypes.c_int64), P(ctypes.c_int32), P(ctypes.c_int32)]
        L.mist_space_destroy.argtypes = [vp]
        L.mist_eval_pareto_exact.argtypes = [vp, vp]
        L.mist_get_pareto_exact.argtypes = [vp, ctypes.c_int64, P(Result), ctypes.c_int64, P(ctypes.c_int64)]
        L.mist_exact_group_sizes.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, P(ctypes.c_int64), P(ctypes.c_int64)]
        L.mist_exact_info.argtypes = [vp, P(ctypes.c_int64), P(ctypes.c_int64), P(ctypes.c_int32), P(ctypes.c_int32)]
        L.mist_plan_points.argtypes = [P(StagePoint), ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, P(Plan)]
        L.mist_plan_pipeline.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, P(Plan)]
        dp = P(ctypes.c_double)
        ip = P(ctypes.c_int32)
        L.mist_corun_create.argtypes = [P(CorunShape), ctypes.c_int32, P(vp)]
        L.mist_corun_run.argtypes = [vp, ctypes.c_int32, P(CorunShape), ip, dp, ctypes.c_int32]
        L.mist_corun_reduce.argtypes = [ctypes.c_int32, dp, ctypes.c_int32, ip, dp, ip]
        L.mist_corun_measure.argtypes = [vp, P(CorunShape), ctypes.c_int32, ctypes.c_double, P(CorunSample),
                                         ctypes.c_int32, ip]
        L.mist_corun_destroy.argtypes = [vp]
        L.mist_fit_phi.argtypes = [P(CorunSample), ctypes.c_int64, dp]
        L.mist_interference.argtypes = [dp, dp, dp]
        L.mist_measure_eta.argtypes = [P(ModelDesc), ip, ctypes.c_int32, ctypes.c_int32, ctypes.c_double,
                                       ctypes.c_int32, dp, dp]
        L.mist_search_info.argtypes = [vp, ip]
        L.mist_tile_info.argtypes = [vp, ctypes.c_int32, P(ctypes.c_int64), P(ctypes.c_uint64), P(ctypes.c_int64)]
        L.mist_debug_eval_tiles.argtypes = [vp, P(ctypes.c_int32), ctypes.c_int32, P(ctypes.c_double),
                                            ctypes.c_int64, vp]
        L.mist_probe_fp64.argtypes = [ctypes.c_int32, vp, vp, ctypes.c_int64, ctypes.c_int32, P(ctypes.c_uint64), vp]
        i32, sz = ctypes.c_int32, ctypes.c_size_t
        L.mist_embed_forward.argtypes = [P(EmbedDesc), vp, vp, vp, vp, vp]
        L.mist_embed_workspace.argtypes = [P(EmbedDesc), P(sz)]
        L.mist_embed_backward.argtypes = [P(EmbedDesc), vp, vp, vp, vp, i32, vp, sz, vp]
        L.mist_tensors_create.argtypes = [P(vp), P(ctypes.c_int64), ctypes.c_int64, i32, P(Allocator), P(vp)]
        L.mist_tensors_destroy.argtypes = [vp]
        L.mist_norm_workspace.argtypes = [vp, P(sz)]
        L.mist_grad_norm.argtypes = [vp, P(ClipDesc), i32, i32, vp, vp, sz, vp]
        L.mist_grad_finish.argtypes = [P(ClipDesc), vp, vp]
        L.mist_grad_clip.argtypes = [vp, vp, vp, vp]
        L.mist_adam_step.argtypes = [vp, vp, vp, vp, vp, vp, P(AdamDesc), vp]
        f32 = ctypes.c_float
        L.mist_token_logprob.argtypes = [P(TokenDesc)] + [vp] * 8
        L.mist_token_part.argtypes = [P(TokenDesc)] + [vp] * 6
        L.mist_token_join.argtypes = [P(TokenDesc), i32] + [vp] * 10
        L.mist_token_grad.argtypes = [P(TokenDesc)] + [vp] * 8
        L.mist_token_loss.argtypes = [P(TokenDesc), vp, vp, vp, f32, vp, vp, vp]
        L.mist_block_forward.argtypes = [P(BlockDesc)] + [vp] * 11
        L.mist_block_workspace.argtypes = [P(BlockDesc), P(BlockGrads), P(sz)]
        L.mist_block_backward.argtypes = [P(BlockDesc)] + [vp] * 7 + [P(BlockGrads), vp, sz, vp]
        L.mist_kept_store.argtypes = [P(KeptDesc)] + [vp] * 4
        L.mist_kept_load.argtypes = [P(KeptDesc)] + [vp] * 4
        L.mist_act_forward.argtypes = [P(ActDesc), vp, vp, vp, P(Kept), P(Kept), vp]
        L.mist_act_backward.argtypes = [P(ActDesc), P(Kept), P(Kept)] + [vp] * 5
        L.mist_last_error.restype = ctypes.c_char_p
        for name in EXPORTS:
            if name != "mist_last_error":
                getattr(L, name).restype = st
        _lib = L
        return L


def _check(L, rc):
    if rc != 0:
        raise MistError(rc, L.mist_last_error().decode())


def _struct_to_dict(s) -> dict:
    out = {}
    for name, _ in s._fields_:
        v = getattr(s, name)
        out[name] = _struct_to_dict(v) if isinstance(v, ctypes.Structure) else v
    return out


def _results_to_dicts(out, n: int) -> list[dict]:
    """mist_result array -> list of dicts, through one numpy view (no per-field ctypes access)."""
    if n == 0:
        return []
    rows = np.ctypeslib.as_array(out)[:n].tolist()
    names = [f for f, _ in Result._fields_[:-1]]
    cnames = [f for f, _ in Config._fields_]
    return [dict(zip(names, r[:-1]), cfg=dict(zip(cnames, r[-1]))) for r in rows]


def _stream_handle(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _torch_allocator(failures: list):
    """PyTorch's caching allocator on the current device as the library's callbacks; the callbacks are
    returned too, to be kept as long as the library may call them."""
    import torch
    device = torch.cuda.current_device()

    def alloc(nbytes, stream, ctx):
        # the block joins the pool of the stream the library uses it on (NULL: the null stream)
        try:
            return torch.cuda.caching_allocator_alloc(int(nbytes), device, int(stream or 0))
        except Exception as e:  # no exception may cross the C ABI
            failures.append(e)
            return None

    def free(ptr, ctx):
        try:
            torch.cuda.caching_allocator_delete(ptr)
        except Exception as e:
            failures.append(e)

    cb = (ALLOC_FN(alloc), FREE_FN(free))
    return Allocator(cb[0], cb[1], None), cb


class Space:
    """A configuration space held by libmist on the current GPU.

    ``model``, ``hws`` and ``space`` are the descriptor dictionaries of
    ``paper_2503_19050_amd.workloads``.  ``allocator="torch"`` routes device memory through
    PyTorch's caching allocator; ``None`` lets the library use hipMalloc.
    """

    def __init__(self, model: dict, hws: list, space: dict, allocator: str | None = "torch"):
        self.L = load()
        self._model = ModelDesc(**{k: model[k] for k, _ in ModelDesc._fields_})
        self._hw = (HwDesc * len(hws))()
        for i, h in enumerate(hws):
            for k in ("flops", "mem_bytes", "pcie_bw", "link_bw", "eta_max", "n_half"):
                setattr(self._hw[i], k, float(h[k]))
            for m in range(16):
                for j in range(4):
                    self._hw[i].phi[m][j] = float(h["phi"][m][j])
            tab = [float(v) for v in h.get("eta_tab", [])]
            self._hw[i].eta_tab[:len(tab)] = tab
        self._mb = np.ascontiguousarray(space["mb"], dtype=np.int32)
        self._ratios = np.ascontiguousarray(space["ratios"], dtype=np.float64)
        self._alphas = np.ascontiguousarray(space.get("alphas", []), dtype=np.float64)
        self.n_alphas = len(self._alphas)
        self._space = SpaceDesc(space["n_devices"], space["global_batch"],
                                self._mb.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), len(self._mb),
                                self._ratios.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                len(self._ratios), space["n_buckets"], space["l_rule"], self.n_alphas,
                                self._alphas.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                int(space.get("tile_configs", 0)), int(space.get("max_blocks", 0)),
                                int(space.get("cand_window", 0)))
        self._alloc = None
        if allocator == "torch":
            self._alloc = self._torch_allocator()
        elif allocator is not None:
            raise ValueError("allocator must be 'torch' or None")
        h = ctypes.c_void_p()
        _check(self.L, self.L.mist_space_create(ctypes.byref(self._model), self._hw, len(hws),
                                                ctypes.byref(self._space),
                                                ctypes.byref(self._alloc) if self._alloc else None,
                                                ctypes.byref(h)))
        self.h = h
        n = ctypes.c_uint64()
        g = ctypes.c_int64()
        nb = ctypes.c_int32()
        _check(self.L, self.L.mist_space_info(self.h, ctypes.byref(n), ctypes.byref(g), ctypes.byref(nb)))
        self.n_configs, self.n_groups, self.n_buckets = n.value, g.value, nb.value

    def _torch_allocator(self):
        self._alloc_failures = []
        allocator, self._cb = _torch_allocator(self._alloc_failures)
        return allocator

    # -- evaluation ---------------------------------------------------------------
    def eval(self, stream=None) -> None:
        """Enqueues the evaluation on ``stream`` (torch stream, raw handle, or current)."""
        _check(self.L, self.L.mist_eval_space(self.h, ctypes.c_void_p(_stream_handle(stream))))

    def set_timing(self, on: bool = True) -> None:
        _check(self.L, self.L.mist_set_timing(self.h, 1 if on else 0))

    def read_timing(self) -> tuple[float, float, int]:
        """(summed evaluation-kernel ms, summed reduction-kernel ms, evaluations) since the
        last read; waits for them."""
        a = ctypes.c_double()
        b = ctypes.c_double()
        n = ctypes.c_int64()
        _check(self.L, self.L.mist_read_timing(self.h, ctypes.byref(a), ctypes.byref(b), ctypes.byref(n)))
        return a.value, b.value, n.value

    def launch_info(self) -> dict:
        t = ctypes.c_int64()
        b = ctypes.c_int32()
        u = ctypes.c_int32()
        _check(self.L, self.L.mist_launch_info(self.h, ctypes.byref(t), ctypes.byref(b), ctypes.byref(u)))
        return {"tiles": t.value, "block": b.value, "strips_per_tile": u.value}

    # -- results ------------------------------------------------------------------
    def best(self, g0: int = 0, n: int | None = None) -> list[dict]:
        n = self.n_groups - g0 if n is None else n
        return _results_to_dicts(self._best_raw(g0, n), n)

    def best_array(self, g0: int = 0, n: int | None = None) -> np.ndarray:
        """best() as a numpy structured array (the mist_result layout), without per-group dicts."""
        n = self.n_groups - g0 if n is None else n
        return np.ctypeslib.as_array(self._best_raw(g0, n))[:n]

    def _best_raw(self, g0: int, n: int):
        out = (Result * max(n, 1)).from_buffer(np.empty(max(n, 1) * ctypes.sizeof(Result), dtype=np.uint8))
        _check(self.L, self.L.mist_get_best(self.h, g0, n, out))
        return out

    def pareto(self, g: int) -> list[dict]:
        out = (Result * 64)()
        cnt = ctypes.c_int32()
        _check(self.L, self.L.mist_get_pareto(self.h, g, out, 64, ctypes.byref(cnt)))
        return _results_to_dicts(out, cnt.value)

    def eval_pareto_exact(self, stream=None) -> None:
        """Exact (non-bucketed) time-vs-memory frontier of every group; after eval()."""
        _check(self.L, self.L.mist_eval_pareto_exact(self.h, _stream_handle(stream)))

    def pareto_exact(self, g: int) -> list[dict]:
        """Group g's exact frontier in increasing memory (strictly decreasing objective)."""
        n = ctypes.c_int64()
        cap = 256
        while True:
            out = (Result * cap)()
            rc = self.L.mist_get_pareto_exact(self.h, g, out, cap, ctypes.byref(n))
            if rc == -5 and n.value > cap:
                cap = n.value
                continue
            _check(self.L, rc)
            return _results_to_dicts(out, n.value)

    def exact_group_sizes(self, g0: int = 0, n: int | None = None) -> tuple[np.ndarray, np.ndarray]:
        """Per-group candidates and pre-filter survivors of the last exact frontier."""
        n = self.n_groups - g0 if n is None else n
        c = np.zeros(max(n, 1), dtype=np.int64)
        k = np.zeros(max(n, 1), dtype=np.int64)
        P = ctypes.POINTER(ctypes.c_int64)
        _check(self.L, self.L.mist_exact_group_sizes(self.h, g0, n, c.ctypes.data_as(P), k.ctypes.data_as(P)))
        return c[:n], k[:n]

    def exact_info(self) -> dict:
        """Sizes of the last exact frontier: candidates, those the pre-filter kept, tiles of the
        candidate pass that may hold one, and tiles evaluated a second time."""
        c, k, v, t = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int32()
        _check(self.L, self.L.mist_exact_info(self.h, ctypes.byref(c), ctypes.byref(k), ctypes.byref(v),
                                              ctypes.byref(t)))
        return {"candidates": c.value, "kept": k.value, "tiles_live": v.value, "tiles_again": t.value}

    def plan(self, hw: int = 0, pp: int = 0) -> dict | None:
        """The inter-stage plan (Eq. 1-3) of hardware sample hw from this space's frontier
        points; pp = 0 allows every stage count.  None when no plan exists."""
        out = Plan()
        _check(self.L, self.L.mist_plan_pipeline(self.h, hw, pp, ctypes.byref(out)))
        return _plan_dict(out)

    def alpha(self, g0: int = 0, n: int | None = None) -> list[list[dict]]:
        """Per group g0..g0+n-1 and weight sample a: the feasible configuration minimising
        alpha_a*G*t + (1-alpha_a)*d (Eq. 4); obj holds that weighted value."""
        n = self.n_groups - g0 if n is None else n
        A = self.n_alphas
        out = (Result * max(n * A, 1))()
        _check(self.L, self.L.mist_get_alpha(self.h, g0, n, out))
        flat = _results_to_dicts(out, n * A)
        return [flat[i * A:(i + 1) * A] for i in range(n)]

    def buckets(self, g0: int = 0, n: int | None = None):
        """(ids[n, NB], objs[n, NB], frontier masks[n]) of groups g0..g0+n-1."""
        n = self.n_groups - g0 if n is None else n
        ids = np.empty((n, self.n_buckets), dtype=np.uint64)
        objs = np.empty((n, self.n_buckets), dtype=np.float64)
        masks = np.empty(n, dtype=np.uint64)
        _check(self.L, self.L.mist_get_buckets(self.h, g0, n,
                                               ids.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)),
                                               objs.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                               masks.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64))))
        return ids, objs, masks

    def eval_ids(self, ids, stream=None) -> np.ndarray:
        """Per-configuration (t, d, mem, obj) computed on the GPU."""
        ids = np.ascontiguousarray(ids, dtype=np.uint64)
        out = np.empty((len(ids), 4), dtype=np.float64)
        _check(self.L, self.L.mist_eval_ids(self.h, ids.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)),
                                            len(ids), out.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                            ctypes.c_void_p(_stream_handle(stream))))
        return out

    def eval_ids_noalloc(self, ids, stream=None) -> np.ndarray:
        """eval_ids through the allocation-free entry point (at most 104,857 ids per call)."""
        ids = np.ascontiguousarray(ids, dtype=np.uint64)
        out = np.empty((len(ids), 4), dtype=np.float64)
        _check(self.L, self.L.mist_eval_ids_noalloc(self.h, ids.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)),
                                                    len(ids), out.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                                    ctypes.c_void_p(_stream_handle(stream))))
        return out

    def searched(self) -> bool:
        """Whether the evaluation searches the space with bounds (else it evaluates every configuration)."""
        b = ctypes.c_int32()
        _check(self.L, self.L.mist_search_info(self.h, ctypes.byref(b)))
        return b.value != 0

    def tile_info(self, t: int) -> dict:
        g = ctypes.c_int64()
        f = ctypes.c_uint64()
        n = ctypes.c_int64()
        _check(self.L, self.L.mist_tile_info(self.h, t, ctypes.byref(g), ctypes.byref(f), ctypes.byref(n)))
        return {"group": g.value, "first_id": f.value, "n_configs": n.value}

    def debug_eval_tiles(self, tiles, stream=None) -> np.ndarray:
        """The evaluation kernel's own per-configuration values over the listed tiles: rows of
        (t, d, mem, obj, bucket entry, forms of Algorithm 1 as f1 + 8 * fs) in tile order, id
        order within a tile."""
        tl = np.ascontiguousarray(tiles, dtype=np.int32)
        total = sum(self.tile_info(int(t))["n_configs"] for t in tl)
        out = np.empty((max(total, 1), 6), dtype=np.float64)
        _check(self.L, self.L.mist_debug_eval_tiles(self.h, tl.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                                    len(tl), out.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                                    total, _stream_handle(stream)))
        return out[:total]

    def decode(self, cid: int) -> dict:
        c = Config()
        _check(self.L, self.L.mist_decode(self.h, cid, ctypes.byref(c)))
        return _struct_to_dict(c)

    def group_key(self, g: int) -> dict:
        k = GroupKey()
        _check(self.L, self.L.mist_get_group_key(self.h, g, ctypes.byref(k)))
        return _struct_to_dict(k)

    def close(self) -> None:
        if getattr(self, "h", None):
            self.L.mist_space_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def from_workload(wl: dict, allocator: str | None = "torch") -> Space:
    return Space(wl["model"], wl["hws"], wl["space"], allocator=allocator)


def plan_points(points, n_layers: int, pp: int = 0) -> dict | None:
    """The host planner on explicit candidate points: an iterable of dicts with keys G, PP, k,
    l, id, t, d.  None when no plan exists."""
    L = load()
    pts = list(points)
    arr = (StagePoint * max(len(pts), 1))()
    for i, p in enumerate(pts):
        arr[i] = StagePoint(p["G"], p["PP"], p["k"], p["l"], p["id"], p["t"], p["d"])
    out = Plan()
    _check(L, L.mist_plan_points(arr, len(pts), n_layers, pp, ctypes.byref(out)))
    return _plan_dict(out)


# -- calibration ------------------------------------------------------------------------------
def _dptr(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_double))


def _iptr(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def _shape(sh: dict) -> CorunShape:
    return CorunShape(*(int(sh[k]) for k, _ in CorunShape._fields_))


def corun_reduce(mask: int, t, units) -> tuple[np.ndarray, np.ndarray]:
    """mist_corun_reduce: t[j] are stream j's timestamps (seconds); returns (mean[4], count[4])."""
    L = load()
    u = np.zeros(4, dtype=np.int32)
    for j in range(4):
        u[j] = units[j]
    stride = int(max([u.max(), 1] + [len(x) - 1 for x in t])) + 1
    tt = np.zeros((4, stride))
    for j in range(4):
        if mask >> j & 1:
            tt[j, :len(t[j])] = t[j]
    mean = np.zeros(4)
    count = np.zeros(4, dtype=np.int32)
    _check(L, L.mist_corun_reduce(int(mask), _dptr(tt), stride, _iptr(u), _dptr(mean), _iptr(count)))
    return mean, count


def fit_phi(samples) -> np.ndarray:
    """mist_fit_phi: samples are (mask, stream, solo_s, corun_s) tuples or dicts; returns phi[16][4]."""
    L = load()
    arr = (CorunSample * max(len(samples), 1))()
    for i, x in enumerate(samples):
        if isinstance(x, dict):
            arr[i] = CorunSample(x["mask"], x["stream"], x.get("shape", 0), x.get("units", 0), x["solo_s"], x["corun_s"])
        else:
            arr[i] = CorunSample(int(x[0]), int(x[1]), 0, 0, float(x[2]), float(x[3]))
    phi = np.zeros(64)
    _check(L, L.mist_fit_phi(arr, len(samples), _dptr(phi)))
    return phi.reshape(16, 4)


def interference(phi, x) -> float:
    """mist_interference: Algorithm 1 on stream times x[4] with factors phi[16][4]."""
    L = load()
    p = np.ascontiguousarray(phi, dtype=np.float64).reshape(64)
    xx = np.ascontiguousarray(x, dtype=np.float64).reshape(4)
    out = ctypes.c_double()
    _check(L, L.mist_interference(_dptr(p), _dptr(xx), ctypes.byref(out)))
    return out.value


def probe_fp64(kind: str, n_threads: int, reps: int, stream=None) -> int:
    """Enqueues the FP64 instruction-mix probe of one kind (add, mul, fma, min, max, cmp) on the
    current (or given) stream; returns the wave-level count of the probed instruction."""
    import torch
    L = load()
    inp = torch.rand(2 * n_threads, dtype=torch.float64, device="cuda") + 0.5
    out = torch.empty(n_threads, dtype=torch.int64, device="cuda")
    n = ctypes.c_uint64()
    _check(L, L.mist_probe_fp64(PROBE_KINDS[kind], ctypes.c_void_p(inp.data_ptr()), ctypes.c_void_p(out.data_ptr()),
                                n_threads, reps, ctypes.byref(n), _stream_handle(stream)))
    torch.cuda.current_stream().synchronize() if stream is None else stream.synchronize()
    return n.value


def measure_eta(model: dict, mb, tp: int, peak_flops: float, reps: int = 5) -> tuple[np.ndarray, np.ndarray]:
    """mist_measure_eta on the current device: (eta[i], seconds[i]) per microbatch size mb[i]."""
    L = load()
    m = ModelDesc(**{k: model[k] for k, _ in ModelDesc._fields_})
    b = np.ascontiguousarray(mb, dtype=np.int32)
    eta = np.zeros(len(b))
    sec = np.zeros(len(b))
    _check(L, L.mist_measure_eta(ctypes.byref(m), _iptr(b), len(b), int(tp), float(peak_flops), int(reps),
                                 _dptr(eta), _dptr(sec)))
    return eta, sec


class Corun:
    """The co-run benchmark's device state (mist_corun_create) on the current device."""

    def __init__(self, max_shape: dict, g2g_blocks: int = 16):
        self.L = load()
        h = ctypes.c_void_p()
        _check(self.L, self.L.mist_corun_create(ctypes.byref(_shape(max_shape)), int(g2g_blocks), ctypes.byref(h)))
        self.h = h

    def run(self, mask: int, shape: dict, units) -> list[np.ndarray]:
        """Timestamps (seconds after the common start) of each member's units."""
        u = np.zeros(4, dtype=np.int32)
        for j in range(4):
            u[j] = units[j]
        stride = CORUN_MAX_UNITS + 1
        t = np.zeros((4, stride))
        _check(self.L, self.L.mist_corun_run(self.h, int(mask), ctypes.byref(_shape(shape)), _iptr(u), _dptr(t),
                                             stride))
        return [t[j, :u[j] + 1].copy() if mask >> j & 1 else np.zeros(0) for j in range(4)]

    def measure(self, shapes, target_s: float = 0.02) -> list[dict]:
        arr = (CorunShape * len(shapes))(*[_shape(s) for s in shapes])
        cap = len(shapes) * CORUN_SAMPLES_PER_SHAPE
        out = (CorunSample * cap)()
        n = ctypes.c_int32()
        _check(self.L, self.L.mist_corun_measure(self.h, arr, len(shapes), float(target_s), out, cap,
                                                 ctypes.byref(n)))
        return [_struct_to_dict(out[i]) for i in range(n.value)]

    def close(self) -> None:
        if getattr(self, "h", None):
            _check(self.L, self.L.mist_corun_destroy(self.h))
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


# -- operators of a training step's two ends ---------------------------------------------------
# They are outside autograd: a gradient is a call of its own, and tensors written in place do not count as
# modified (their version counters stay).
E_INVALID = -1
_NORMS = {"l2": 0, "max": 1}
NORM_WORKSPACE = 16384
_TYPES = {}  # torch dtype -> element type


def _torch():
    import torch
    if not _TYPES:
        _TYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    return torch


def _need(ok: bool, msg: str) -> None:
    if not ok:
        raise MistError(E_INVALID, msg)


def _type(t, what: str) -> int:
    code = _TYPES.get(t.dtype)
    _need(code is not None, "%s: %s is not float32, bfloat16 or float16" % (what, t.dtype))
    return code


def _stream_of(torch, stream, device):
    """A caller's stream (None, raw handle or torch stream) as (handle, torch stream or None)."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index), None
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
    _need(stream.device == device, "the stream is of another device than the tensors")
    return stream.cuda_stream, stream


def _on_device(torch, device, fn, *args) -> None:
    """One call of the library with the tensors' device current."""
    if torch._C._cuda_getDevice() == device.index:
        _check(_lib, fn(*args))
    else:
        with torch.cuda.device(device):
            _check(_lib, fn(*args))


def _used_on(stream, *tensors) -> None:
    """Tells the caching allocator that the tensors are used on a stream other than the current one."""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def _embed_desc(ids, act, table, scale, pos, vocab_begin) -> EmbedDesc:
    device = act.device
    _need(act.is_cuda and ids.device == device and table.device == device and (pos is None or pos.device == device),
          "embedding: ids, table, positions and activations must be on one GPU")
    id_bytes = ids.element_size()
    _need(id_bytes in (4, 8) and not ids.dtype.is_floating_point and not ids.dtype.is_complex and ids.dtype.is_signed,
          "embedding: ids must be int32 or int64")
    shape, ashape = ids.shape, act.shape
    dims = len(shape)
    _need(dims in (1, 2) and len(ashape) == dims + 1 and ashape[:-1] == shape,
          "embedding: ids must be [seq] or [batch, seq], the activations ids' shape and hidden")
    seq, hidden, tshape = shape[-1], ashape[-1], table.shape
    _need(len(tshape) == 2 and tshape[1] == hidden, "embedding: the table must be [rows, hidden]")
    ist, ast, tst = ids.stride(), act.stride(), table.stride()
    _need(hidden == 1 or ((ast[-1] == 1 or act.numel() == 0) and tst[1] == 1), "embedding: the hidden dimension must be contiguous")
    _need(seq <= 1 or ist[-1] == 1, "embedding: the ids of a sequence must be contiguous")
    pos_stride = 0
    if pos is not None:
        _need(pos.dim() == 2 and pos.shape[1] == hidden and pos.shape[0] >= seq, "embedding: the positions must be [at least seq, hidden]")
        _need(pos.dtype == table.dtype, "embedding: the positions must have the table's type")
        pst = pos.stride()
        _need(hidden == 1 or pst[1] == 1 or pos.numel() == 0, "embedding: the hidden dimension must be contiguous")
        pos_stride = pst[0]
    two = dims == 2
    return EmbedDesc(shape[0] if two else 1, seq, hidden, tshape[0], int(vocab_begin), ist[0] if two else 0, ast[0] if two else 0,
                     ast[-2], tst[0], pos_stride, id_bytes, _type(act, "embedding"), _type(table, "embedding"), float(scale))


def _ptr(t):
    return None if t is None else t.data_ptr()


def embed(ids, table, *, scale: float = 1.0, pos=None, vocab_begin: int = 0, out=None, stream=None):
    """mist_embed_forward: scale * table[ids - vocab_begin] + pos[position], zero in the first term for ids
    outside the shard (padding, other ranks' rows).  ids: [seq] or [batch, seq], int32 or int64 (batch strides
    allowed); table: [rows, hidden]; pos: [at least seq, hidden] or None; out: ids' shape + [hidden], of
    any of float32, bfloat16, float16 (default: a new tensor of the table's type).  Ranks that hold shards of the
    table add up what they get: one of them passes pos, the others None."""
    torch = _torch()
    L = _lib or load()
    if (table.requires_grad or pos is not None and pos.requires_grad) and torch.is_grad_enabled():
        _need(False, "embedding: records no gradient; call it under torch.no_grad() and embed_grad for the gradients")
    if not table.is_cuda:
        _need(False, "embedding: ids, table, positions and activations must be on one GPU")
    handle, other = _stream_of(torch, stream, table.device)
    if out is None:
        _need(table.dim() == 2, "embedding: the table must be [rows, hidden]")
        with torch.cuda.stream(other):
            out = torch.empty(tuple(ids.shape) + (table.shape[1],), dtype=table.dtype, device=table.device)
    d = _embed_desc(ids, out, table, scale, pos, vocab_begin)
    _on_device(torch, out.device, L.mist_embed_forward, ctypes.byref(d), ids.data_ptr(), table.data_ptr(), _ptr(pos),
               out.data_ptr(), handle)
    if other is not None:
        _used_on(other, ids, table, pos, out)
    return out


def embed_grad(ids, grad, dtable, *, scale: float = 1.0, dpos=None, vocab_begin: int = 0, accumulate: bool = False,
               stream=None):
    """mist_embed_backward: the gradients of embed's table and positions from grad (ids' shape + [hidden]; it
    may be expanded), written to dtable and dpos (accumulate: added to them)."""
    torch = _torch()
    L = _lib or load()
    d = _embed_desc(ids, grad, dtable, scale, dpos, vocab_begin)
    device = grad.device
    handle, other = _stream_of(torch, stream, device)
    need = ctypes.c_size_t()
    _check(L, L.mist_embed_workspace(ctypes.byref(d), ctypes.byref(need)))
    if other is None:
        ws = torch.empty(need.value, dtype=torch.uint8, device=device)
    else:
        with torch.cuda.stream(other):  # of that stream's pool
            ws = torch.empty(need.value, dtype=torch.uint8, device=device)
    _on_device(torch, device, L.mist_embed_backward, ctypes.byref(d), ids.data_ptr(), grad.data_ptr(), dtable.data_ptr(), _ptr(dpos),
               1 if accumulate else 0, ws.data_ptr(), need.value, handle)
    if other is not None:
        _used_on(other, ids, grad, dtable, dpos)
    return dtable


_closed = []  # lists that wait to be freed: (library, handle, callbacks)


def _free_closed(torch) -> None:
    """Frees closed lists, which waits for the device: not while a graph is captured, whose capture that would end."""
    if torch.cuda.is_current_stream_capturing():
        return
    for _ in range(len(_closed)):
        entry = _closed.pop()
        if entry[0].mist_tensors_destroy(entry[1]) != 0:
            _closed.insert(0, entry)


class TensorList:
    """Tensors of one type on the current GPU as one list (mist_tensors_create), e.g. a stage's gradients.  They
    must be contiguous and stay where they are; the list keeps them alive.  One that holds a value twice (tied weights listed
    under both names) can be read but not written.  Making a list copies its tables to the
    device and waits, closing it waits for the device: lists are for tensors that stay over many steps.  No list is
    made while a graph is captured, one that is closed then is freed later; a graph needs its lists as long as it is replayed."""

    def __init__(self, tensors, allocator: str | None = "torch"):
        self.h = None
        torch = _torch()
        self.L = load()
        self.tensors = list(tensors)
        _need(len(self.tensors) > 0, "tensor list: no tensors")
        _need(allocator in ("torch", None), "allocator must be 'torch' or None")
        t0 = self.tensors[0]
        self.dtype, self.device = t0.dtype, t0.device
        for t in self.tensors:
            _need(t.is_cuda and t.device == self.device and t.dtype == self.dtype,
                  "tensor list: the tensors must be of one type on one GPU")
            _need(t.is_contiguous(), "tensor list: the tensors must be contiguous")
        code = _type(t0, "tensor list")
        n = len(self.tensors)
        ptrs = (ctypes.c_void_p * n)(*[t.data_ptr() for t in self.tensors])
        sizes = (ctypes.c_int64 * n)(*[t.numel() for t in self.tensors])
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _need(not torch.cuda.is_current_stream_capturing(), "tensor list: cannot be made while a graph is captured")
            _free_closed(torch)
            self._alloc = None
            if allocator == "torch":
                self._alloc, self._cb = _torch_allocator([])
            _check(self.L, self.L.mist_tensors_create(ptrs, sizes, n, code, ctypes.byref(self._alloc) if self._alloc else None,
                                                      ctypes.byref(h)))
        self.h = h

    def __len__(self) -> int:
        return len(self.tensors)

    def close(self) -> None:
        if getattr(self, "h", None):
            h, self.h = self.h, None
            _closed.append((self.L, h, getattr(self, "_cb", None)))
            _free_closed(_torch())

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class StepRecord:
    """A mist_step_record on the GPU, with the norm's scratch memory behind it; the fields are 0-dimensional tensors
    that share its memory.  One stream at a time."""

    def __init__(self, step: int = 0, device=None):
        torch = _torch()
        _need(step >= 0, "step record: step must be >= 0")
        _need(device is None or torch.device(device).type == "cuda", "step record: must be on a GPU")
        self.data = torch.zeros(8 + NORM_WORKSPACE // 8, dtype=torch.float64, device="cuda" if device is None else device)
        self.device = self.data.device
        self.ptr = self.data.data_ptr()
        self.total = self.data[0]
        self.step = self.data.view(torch.int64)[1]
        f, i = self.data.view(torch.float32), self.data.view(torch.int32)
        self.norm, self.coef = f[4], f[5]
        self.applied, self.skipped = i[6], i[7]
        if step:
            self.step.fill_(int(step))


def _clip_desc(kind, grad_scale, max_norm) -> ClipDesc:
    _need(kind in _NORMS, "gradient norm: kind must be 'l2' or 'max'")
    return ClipDesc(_NORMS[kind], grad_scale, max_norm)


def _lists_on(record, *lists) -> None:
    for x in lists:
        _need(x.h is not None, "tensor list: closed")
        _need(x.device == record.device, "tensor list: on another device than the step record")


def grad_norm(grads: TensorList, record: StepRecord, *, max_norm: float = float("inf"), grad_scale: float = 1.0, kind: str = "l2",
              accumulate: bool = False, finish: bool = True, stream=None) -> StepRecord:
    """mist_grad_norm over a list: record.total, and with finish the norm, the clip factor and the count of
    the step.  Nothing is waited for.  accumulate joins record.total (a step with several lists).  Where ranks add
    up their totals, a tensor that several of them hold is in one rank's list alone."""
    torch = _torch()
    c = _clip_desc(kind, grad_scale, max_norm)
    _lists_on(record, grads)
    handle, other = _stream_of(torch, stream, record.device)
    _on_device(torch, record.device, grads.L.mist_grad_norm, grads.h, ctypes.byref(c), 1 if accumulate else 0, 1 if finish else 0,
               record.ptr, record.ptr + 64, NORM_WORKSPACE, handle)
    if other is not None:
        _used_on(other, record.data, *grads.tensors)
    return record


def grad_finish(record: StepRecord, *, max_norm: float = float("inf"), grad_scale: float = 1.0, kind: str = "l2",
                stream=None) -> StepRecord:
    """mist_grad_finish: forms the norm and the clip factor from record.total, e.g. after an all-reduce of it.  With
    record.total.zero_() before it, a step without a pass over the gradients: the factor is grad_scale."""
    torch = _torch()
    L = _lib or load()
    c = _clip_desc(kind, grad_scale, max_norm)
    handle, other = _stream_of(torch, stream, record.device)
    _on_device(torch, record.device, L.mist_grad_finish, ctypes.byref(c), record.ptr, handle)
    if other is not None:
        _used_on(other, record.data)
    return record


def grad_clip(grads: TensorList, record: StepRecord, out: TensorList | None = None, *, stream=None) -> None:
    """mist_grad_clip: out = record.coef * grads (out None: in place)."""
    torch = _torch()
    out = grads if out is None else out
    _lists_on(record, grads, out)
    handle, other = _stream_of(torch, stream, record.device)
    _on_device(torch, record.device, grads.L.mist_grad_clip, grads.h, record.ptr, out.h, handle)
    if other is not None:
        _used_on(other, record.data, *grads.tensors, *out.tensors)


def adam_step(master: TensorList, m: TensorList, v: TensorList, grads: TensorList, record: StepRecord, *, lr: float,
              betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0, weights: TensorList | None = None,
              stream=None) -> None:
    """mist_adam_step with record's clip factor and step count; weights receives the rounded master weights."""
    torch = _torch()
    lists = (master, m, v, grads) if weights is None else (master, m, v, grads, weights)
    _lists_on(record, *lists)
    a = AdamDesc(lr, betas[0], betas[1], eps, weight_decay)
    handle, other = _stream_of(torch, stream, record.device)
    _on_device(torch, record.device, grads.L.mist_adam_step, master.h, m.h, v.h, grads.h, None if weights is None else weights.h,
               record.ptr, ctypes.byref(a), handle)
    if other is not None:
        _used_on(other, record.data, *(t for x in lists for t in x.tensors))


# ---- the last stage and a layer beside its matrix products: loss, norms, kept activations ---------------
TOKEN_MAX_TOP = 64
KEPT_GROUP = 128
_BLOCK_KINDS = {"rms": 0, "layer": 1}
_ACTS = {"silu": 0, "gelu": 1}

TokenLogprob = collections.namedtuple("TokenLogprob", "logp lse entropy top_ids top_logp")
TokenPart = collections.namedtuple("TokenPart", "stats top_ids top_z")
BlockNorm = collections.namedtuple("BlockNorm", "y h stats")
MlpAct = collections.namedtuple("MlpAct", "out up gate")


def _no_graph(torch, what, *tensors) -> None:
    forward = torch.autograd.forward_ad
    if forward._current_level >= 0:   # forward mode, also under no_grad
        for t in tensors:
            if t is not None and forward.unpack_dual(t).tangent is not None:
                _need(False, "%s: has no forward-mode gradient; a tensor with a tangent is given" % what)
    if not torch.is_grad_enabled():
        return
    for t in tensors:
        if t is not None and t.requires_grad:
            _need(False, "%s: records no gradient; call it under torch.no_grad() and the gradient's call for the gradients" % what)


def _here(what, first, *tensors) -> None:
    device = first.device
    for t in tensors:
        if t is not None and t.device != device:
            device = None
            break
    if device is None or not first.is_cuda:
        _need(False, "%s: the tensors must be on one GPU" % what)


class _Idle:
    def __enter__(self):
        return self

    def __exit__(self, *exc):
        return None


_IDLE = _Idle()


def _pool(torch, other):
    """New tensors of the pool of the stream that they are used on (other; None: the current one)."""
    return _IDLE if other is None else torch.cuda.stream(other)


def _like(torch, t, dtype=None):
    """A new contiguous tensor of t's shape."""
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def _shaped(what, t, shape, dtype, name) -> None:
    if not (t.dtype == dtype and t.shape == shape):
        _need(False, "%s: %s must be %s of %s" % (what, name, dtype, tuple(shape)))


def _flat(what, t) -> tuple[int, int]:
    """(rows, their stride) of a tensor whose last dimension is contiguous and whose others are rows at one stride."""
    shape, strides = t.shape, t.stride()
    if not (len(shape) >= 1):
        _need(False, "%s: a tensor without dimensions" % what)
    if t.is_contiguous():
        width = shape[-1]
        return (t.numel() // width if width else 0), width
    rows, stride = 1, shape[-1]
    if t.numel() == 0:
        return 0, stride
    if not (shape[-1] == 1 or strides[-1] == 1):
        _need(False, "%s: the last dimension must be contiguous" % what)
    for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n == 1:
            continue
        if rows == 1:
            stride = s
        if not (s == stride * rows):
            _need(False, "%s: the leading dimensions must be rows at one stride" % what)
        rows *= n
    return rows, stride


def _packed(what, t, shape, dtype, name):
    _shaped(what, t, shape, dtype, name)
    if not (t.is_contiguous()):
        _need(False, "%s: %s must be contiguous" % (what, name))
    return t


def _targets(what, targets, shape) -> tuple[int, int]:
    """(stride between sequences, bytes of an id) of targets for tokens of this shape."""
    if targets is None:
        return 0, 8
    id_bytes, dtype = targets.element_size(), targets.dtype
    if not (id_bytes in (4, 8) and not dtype.is_floating_point and not dtype.is_complex and dtype.is_signed):
        _need(False, "%s: targets must be int32 or int64" % what)
    if targets.shape != shape:
        _need(False, "%s: targets must have the logits' shape but for the last dimension" % what)
    strides = targets.stride()
    if not (shape[-1] <= 1 or strides[-1] == 1):
        _need(False, "%s: the targets of a sequence must be contiguous" % what)
    return strides[0] if len(shape) == 2 else 0, id_bytes


def _token_desc(torch, logits, targets, grad, vocab_begin, scale, top) -> TokenDesc:
    what = "token log probabilities"
    _here(what, logits, targets, grad)
    shape, lst = logits.shape, logits.stride()
    dims, rows = len(shape), shape[-1] if len(shape) else 0
    if dims != 3 and dims != 2:
        _need(False, "%s: the logits must be [seq, rows] or [batch, seq, rows]" % what)
    ist, id_bytes = _targets(what, targets, shape[:-1])
    if not (rows <= 1 or lst[-1] == 1 or logits.numel() == 0):
        _need(False, "%s: the last dimension must be contiguous" % what)
    gst = lst
    if grad is not None:
        if not (grad.shape == shape and grad.dtype == logits.dtype):
            _need(False, "%s: the gradient must have the logits' shape and type" % what)
        gst = grad.stride()
        if not (rows <= 1 or gst[-1] == 1 or logits.numel() == 0):
            _need(False, "%s: the last dimension must be contiguous" % what)
    code = _type(logits, what)
    if dims == 3:
        return TokenDesc(shape[0], shape[1], rows, vocab_begin, ist, lst[0], lst[1], gst[0], gst[1], id_bytes, code, top, scale)
    return TokenDesc(1, shape[0], rows, vocab_begin, ist, 0, lst[0], 0, gst[0], id_bytes, code, top, scale)


def _top_space(torch, shape, top, device):
    if not top:
        return None, None
    if not (0 < top <= TOKEN_MAX_TOP):
        _need(False, "token log probabilities: top must be in 0..%d" % TOKEN_MAX_TOP)
    ids = torch.empty(shape + (top,), dtype=torch.int32, device=device)
    return ids, torch.empty_like(ids, dtype=torch.float32)


def token_logprob(logits, targets=None, *, scale: float = 1.0, entropy: bool = False, top: int = 0, stream=None) -> TokenLogprob:
    """mist_token_logprob over the whole vocabulary: fp32 logp of the targets (None without them; 0 for padding, targets below 0),
    lse, entropy (None if not asked for), and the `top` most probable ids with their log probabilities.  logits: [seq, vocab] or
    [batch, seq, vocab] (strides allowed, e.g. without the last position), scale 1 / temperature; targets: int32 or int64."""
    torch = _torch()
    L = _lib or load()
    _no_graph(torch, "token log probabilities", logits)
    d = _token_desc(torch, logits, targets, None, 0, scale, top)
    device, shape = logits.device, tuple(logits.shape[:-1])
    handle, other = _stream_of(torch, stream, device)
    with _pool(torch, other):
        lse = torch.empty(shape, dtype=torch.float32, device=device)
        logp = None if targets is None else torch.empty_like(lse)
        ent = torch.empty_like(lse) if entropy else None
        ids, values = _top_space(torch, shape, top, device)
    _on_device(torch, device, L.mist_token_logprob, ctypes.byref(d), logits.data_ptr(), _ptr(targets), _ptr(logp), lse.data_ptr(), _ptr(ent),
               _ptr(ids), _ptr(values), handle)
    if other is not None:
        _used_on(other, logits, targets)
    return TokenLogprob(logp, lse, ent, ids, values)


def token_part(logits, targets, *, vocab_begin: int, scale: float = 1.0, top: int = 0, stats=None, stream=None) -> TokenPart:
    """mist_token_part: what a rank with the logits of ids [vocab_begin, vocab_begin + rows) knows of each token, for
    token_join over all ranks' (all-gathered) parts: stats [..., 4] (given, e.g. this rank's place in what is gathered, or
    new) and its `top` alternatives.  targets are ids of the whole vocabulary."""
    torch = _torch()
    L = _lib or load()
    if targets is None:
        _need(False, "token log probabilities: a part needs targets")
    _no_graph(torch, "token log probabilities", logits)
    d = _token_desc(torch, logits, targets, None, vocab_begin, scale, top)
    device, shape = logits.device, tuple(logits.shape[:-1])
    handle, other = _stream_of(torch, stream, device)
    with _pool(torch, other):
        if stats is None:
            stats = torch.empty(shape + (4,), dtype=torch.float32, device=device)
        ids, z = _top_space(torch, shape, top, device)
    _here("token log probabilities", logits, stats)
    _packed("token log probabilities", stats, shape + (4,), torch.float32, "stats")
    _on_device(torch, device, L.mist_token_part, ctypes.byref(d), logits.data_ptr(), targets.data_ptr(), stats.data_ptr(), _ptr(ids), _ptr(z), handle)
    if other is not None:
        _used_on(other, logits, targets, stats)
    return TokenPart(stats, ids, z)


def token_join(stats, targets=None, *, entropy: bool = False, top_ids=None, top_z=None, stream=None) -> TokenLogprob:
    """mist_token_join: token_logprob's results from the parts of all ranks, stats [ranks, ..., 4], and top_ids and top_z
    [ranks, ..., top] where alternatives are wanted (in the order of z, the lower id first among equals)."""
    torch = _torch()
    L = _lib or load()
    what = "token log probabilities"
    if not (stats.dim() in (3, 4) and stats.shape[-1] == 4):
        _need(False, "%s: stats must be [ranks, seq, 4] or [ranks, batch, seq, 4]" % what)
    _here(what, stats, targets, top_ids, top_z)
    ranks, shape, device = stats.shape[0], tuple(stats.shape[1:-1]), stats.device
    _packed(what, stats, stats.shape, torch.float32, "stats")
    top = 0
    if not ((top_ids is None) == (top_z is None)):
        _need(False, "%s: top_ids and top_z come together" % what)
    if top_ids is not None:
        top = top_ids.shape[-1]
        _packed(what, top_ids, (ranks,) + shape + (top,), torch.int32, "top_ids")
        _packed(what, top_z, (ranks,) + shape + (top,), torch.float32, "top_z")
    ist, id_bytes = _targets(what, targets, shape)
    d = TokenDesc(shape[0] if len(shape) == 2 else 1, shape[-1], 1, 0, ist, 0, 0, 0, 0, id_bytes, 0, top, 1.0)
    handle, other = _stream_of(torch, stream, device)
    with _pool(torch, other):
        lse = torch.empty(shape, dtype=torch.float32, device=device)
        logp = None if targets is None else torch.empty_like(lse)
        ent = torch.empty_like(lse) if entropy else None
        ids, values = _top_space(torch, shape, top, device)
    _on_device(torch, device, L.mist_token_join, ctypes.byref(d), ranks, stats.data_ptr(), _ptr(top_ids), _ptr(top_z), _ptr(targets), _ptr(logp),
               lse.data_ptr(), _ptr(ent), _ptr(ids), _ptr(values), handle)
    if other is not None:
        _used_on(other, stats, targets, top_ids, top_z)
    return TokenLogprob(logp, lse, ent, ids, values)


def token_grad(logits, targets, lse, *, dlogp=None, entropy=None, dentropy=None, vocab_begin: int = 0, scale: float = 1.0, dlogits=None,
               stream=None):
    """mist_token_grad: the logits' gradient from those of logp and entropy (fp32 per token; None: zero), with lse and entropy of the
    whole vocabulary.  dlogits: of the logits' shape and type (it may be the logits; default: a new tensor)."""
    torch = _torch()
    L = _lib or load()
    what = "token log probabilities' gradient"
    _here(what, logits, lse, dlogp, entropy, dentropy, targets, dlogits)
    if not (logits.dim() in (2, 3)):
        _need(False, "%s: the logits must be [seq, rows] or [batch, seq, rows]" % what)
    handle, other = _stream_of(torch, stream, logits.device)
    if dlogits is None:
        with _pool(torch, other):
            dlogits = _like(torch, logits)
    if not (dlogp is None or targets is not None):
        _need(False, "%s: dlogp without targets" % what)
    if not (dentropy is None or entropy is not None):
        _need(False, "%s: dentropy without entropy" % what)
    d = _token_desc(torch, logits, targets, dlogits, vocab_begin, scale, 0)
    for t, name in ((lse, "lse"), (dlogp, "dlogp"), (entropy, "entropy"), (dentropy, "dentropy")):
        if t is not None:
            _packed(what, t, logits.shape[:-1], torch.float32, name)
    _on_device(torch, logits.device, L.mist_token_grad, ctypes.byref(d), logits.data_ptr(), _ptr(targets), lse.data_ptr(), _ptr(dlogp), _ptr(entropy),
               _ptr(dentropy), dlogits.data_ptr(), handle)
    if other is not None:
        _used_on(other, logits, targets, lse, dlogp, entropy, dentropy, dlogits)
    return dlogits


def token_loss(logits, targets, weights=1.0, *, scale: float = 1.0, dlogits=None, stream=None):
    """mist_token_loss, a training microbatch in one pass: (logp, dlogits) with dlogits the gradient of the loss
    -sum(weights * logp).  weights: fp32 per token, or one number (1 / tokens for a mean).  dlogits as in token_grad."""
    torch = _torch()
    L = _lib or load()
    what = "token loss"
    if targets is None:
        _need(False, "token loss: needs targets")
    _no_graph(torch, what, logits)
    _here(what, logits, targets, dlogits)
    if not (logits.dim() in (2, 3)):
        _need(False, "%s: the logits must be [seq, rows] or [batch, seq, rows]" % what)
    device, shape = logits.device, logits.shape[:-1]
    w, factor = (weights, 1.0) if isinstance(weights, torch.Tensor) else (None, float(weights))
    if w is not None:
        _here(what, logits, w)
        _packed(what, w, shape, torch.float32, "weights")
    handle, other = _stream_of(torch, stream, device)
    with _pool(torch, other):
        if dlogits is None:
            dlogits = _like(torch, logits)
        logp = torch.empty(shape, dtype=torch.float32, device=device)
    d = _token_desc(torch, logits, targets, dlogits, 0, scale, 0)
    _on_device(torch, device, L.mist_token_loss, ctypes.byref(d), logits.data_ptr(), targets.data_ptr(), _ptr(w), factor, logp.data_ptr(),
               dlogits.data_ptr(), handle)
    if other is not None:
        _used_on(other, logits, targets, w, dlogits)
    return logp, dlogits


def _block_weights(what, hidden, dtype, *weights) -> None:
    for t in weights:
        if t is not None and not (t.dtype is dtype and t.dim() == 1 and t.shape[0] == hidden and t.is_contiguous()):
            _need(False, "%s: weights and biases must be [%d] of one type, contiguous" % (what, hidden))


def _block_gate(what, x, gate, dtype) -> int:
    """The stride between sequences' gates."""
    hidden = x.shape[-1]
    if not (gate.dtype == dtype and (tuple(gate.shape) == (hidden,) or (x.dim() == 3 and tuple(gate.shape) == (x.shape[0], hidden)))):
        _need(False, "%s: the gate must be [hidden], or [batch, hidden] for [batch, seq, hidden], of the weights' type" % what)
    if not (hidden <= 1 or gate.stride(-1) == 1):
        _need(False, "%s: the last dimension must be contiguous" % what)
    return gate.stride(0) if gate.dim() == 2 else 0


def _block_desc(what, x, block, y, h, weight, bias, post_weight, post_bias, gate, kind, eps, res_scale, block_scale, of_sum=0):
    shape = x.shape
    dims, hidden = len(shape), shape[-1] if len(shape) else 0
    if dims != 3 and dims != 2:
        _need(False, "%s: must be [tokens, hidden] or [batch, seq, hidden]" % what)
    code = _BLOCK_KINDS.get(kind)
    if code is None:
        _need(False, "%s: kind must be 'rms' or 'layer'" % what)
    like = block if block is not None else h if h is not None else x
    first = weight if weight is not None else post_weight if post_weight is not None else bias if bias is not None else post_bias
    first = first if first is not None else gate
    rtype = x.dtype
    wtype = rtype if first is None else first.dtype
    if weight is not None or post_weight is not None or bias is not None or post_bias is not None:
        _block_weights(what, hidden, wtype, weight, bias, post_weight, post_bias)
    strides = [hidden if x.is_contiguous() else _flat(what, x)[1], 0, 0, 0]
    for k, t in ((1, block), (2, y), (3, h)):
        if t is not None and t is not x:
            if t.shape != shape:
                _need(False, "%s: the tensors must have one shape" % what)
            strides[k] = hidden if t.is_contiguous() else _flat(what, t)[1]
        elif t is x:
            strides[k] = strides[0]
    if y is not None and y.dtype != rtype:
        _need(False, "%s: y must have x's type" % what)
    if h is not None and h.dtype != like.dtype:
        _need(False, "%s: h must have the block's type" % what)
    return BlockDesc(shape[0] if dims == 3 else 1, shape[-2], hidden, strides[0], strides[1], strides[2], strides[3],
                     0 if gate is None else _block_gate(what, x, gate, wtype), code, _type(like, what), _type(x, what), _TYPES.get(wtype, -1),
                     eps, res_scale, block_scale, of_sum)


def block_norm(x, block=None, *, weight=None, bias=None, post_weight=None, post_bias=None, gate=None, kind: str = "rms", eps: float = 1e-6,
               res_scale: float = 1.0, block_scale: float = 1.0, stored: bool = True, y=None, h=None, dtype=None, stream=None) -> BlockNorm:
    """mist_block_forward: y = res_scale * x + block_scale * gate * N(block), h = N(y) * weight + bias, and the stats that
    block_norm_grad takes.  x: [tokens, hidden] or [batch, seq, hidden], the residual, of the block's type or float32; gate: [hidden]
    or [batch, hidden].  Without post_weight the block's output is not normed; without weight there is no h (None); without
    block, y is x and h its norm (of dtype, default x's).  stored: N(y) is of y as it is stored, so that block_norm of y alone gives h bit
    for bit; False: of the sum before its rounding, so that h of a 16-bit residual has one rounding, not two.  y may be x or block."""
    torch = _torch()
    L = _lib or load()
    what = "block norm"
    _no_graph(torch, what, x, block, weight, bias, post_weight, post_bias, gate)
    _here(what, x, block, weight, bias, post_weight, post_bias, gate, y, h)
    handle, other = _stream_of(torch, stream, x.device)
    if not (block is None or dtype is None or dtype == block.dtype):
        _need(False, "block norm: dtype is the block's")
    if not (block is not None or y is None):
        _need(False, "block norm: without a block y is x")
    if not (weight is not None or h is None):
        _need(False, "block norm: h without its weight")
    with _pool(torch, other):
        if block is not None and y is None:
            y = _like(torch, x)
        if weight is not None and h is None:
            h = _like(torch, x, dtype if block is None else block.dtype)
        stats = torch.empty((*x.shape[:-1], 4), dtype=torch.float32, device=x.device)
    d = _block_desc(what, x, block, y, h, weight, bias, post_weight, post_bias, gate, kind, eps, res_scale, block_scale, 0 if stored else 1)
    _on_device(torch, x.device, L.mist_block_forward, ctypes.byref(d), x.data_ptr(), _ptr(block), _ptr(weight), _ptr(bias), _ptr(post_weight),
               _ptr(post_bias), _ptr(gate), _ptr(y), _ptr(h), stats.data_ptr(), handle)
    if other is not None:
        _used_on(other, x, block, weight, bias, post_weight, post_bias, gate, y, h)
    return BlockNorm(x if y is None else y, h, stats)


def block_norm_grad(y, stats, dh=None, *, block=None, dy=None, weight=None, post_weight=None, post_bias=None, gate=None, kind: str = "rms",
                    res_scale: float = 1.0, block_scale: float = 1.0, dweight=None, dbias=None, dpost_weight=None, dpost_bias=None, dgate=None,
                    accumulate: bool = False, dx=None, dblock=None, stream=None):
    """mist_block_backward: (dx, dblock) from dh and dy (the gradient of y by its other uses; None: none), with y and stats of
    block_norm and its arguments.  Gradients of weights, biases and gates go to the given tensors of the weights' type
    (accumulate: added to them).  dx may be dy, dblock may be dh or block; by default they are new."""
    torch = _torch()
    L = _lib or load()
    what = "block norm's gradient"
    grads = (dweight, dbias, dpost_weight, dpost_bias)
    _here(what, y, stats, dh, block, dy, weight, post_weight, post_bias, gate, *grads, dgate, dx, dblock)
    handle, other = _stream_of(torch, stream, y.device)
    if not (dh is not None or dy is not None):
        _need(False, "%s: neither dh nor dy" % what)
    if not ((dh is None) == (weight is None)):
        _need(False, "%s: dh comes with weight" % what)
    if not (block is not None or dblock is None):
        _need(False, "%s: of a block that is not there" % what)
    with _pool(torch, other):
        if dx is None:
            dx = _like(torch, y)
        if block is not None and dblock is None:
            dblock = _like(torch, block)
    shared = gate
    if gate is not None and dgate is not None and gate.dim() == 2 and gate.shape[0] > 1 and gate.stride(0) == 0:
        with _pool(torch, other):  # rows of one place: their gradients are still a row for each sequence
            gate = gate.contiguous()
    d = _block_desc(what, y, block, y, dh, weight, None, post_weight, post_bias, gate, kind, 0.0, res_scale, block_scale)
    first = weight if weight is not None else post_weight if post_weight is not None else gate
    wtype = y.dtype if first is None else first.dtype
    _block_weights(what, y.shape[-1], wtype, *grads)
    dgate_stride = 0
    if dgate is not None:
        if not (gate is not None and dgate.shape == gate.shape):
            _need(False, "%s: dgate must have the gate's shape" % what)
        dgate_stride = _block_gate(what, y, dgate, wtype)
    shape, rtype = y.shape, y.dtype
    _packed(what, stats, (*shape[:-1], 4), torch.float32, "stats")
    strides, btype = [], None if block is None else block.dtype
    for t, dtype in ((dh, btype), (dy, rtype), (dx, rtype), (dblock, btype)):
        if t is None:
            strides.append(0)
            continue
        if t.shape != shape or (dtype is not None and t.dtype != dtype):
            _need(False, "%s: a gradient must have its tensor's shape and type" % what)
        strides.append(shape[-1] if t.is_contiguous() else _flat(what, t)[1])
    g = BlockGrads(_ptr(dh), _ptr(dy), _ptr(dx), _ptr(dblock), *(_ptr(t) for t in grads), _ptr(dgate), *strides, dgate_stride, 1 if accumulate else 0)
    need = ctypes.c_size_t()
    _check(L, L.mist_block_workspace(ctypes.byref(d), ctypes.byref(g), ctypes.byref(need)))
    ws = None
    if need.value:
        with _pool(torch, other):  # of that stream's pool
            ws = torch.empty(need.value, dtype=torch.uint8, device=y.device)
    _on_device(torch, y.device, L.mist_block_backward, ctypes.byref(d), y.data_ptr(), _ptr(block), stats.data_ptr(), _ptr(weight), _ptr(post_weight),
               _ptr(post_bias), _ptr(gate), ctypes.byref(g), _ptr(ws), need.value, handle)
    if other is not None:
        _used_on(other, y, stats, dh, block, dy, weight, post_weight, post_bias, shared, *grads, dgate, dx, dblock)
    return dx, dblock


class Checkpoint:
    """A tensor kept in 8 bits (mist_kept_store): int8 values and uint8 exponents, a byte for each 128 values of a row, both plain tensors
    that a program can offload or send.  shape and dtype are the tensor's; stream: the one that it is used on (None: the current one)."""

    def __init__(self, shape, dtype, device="cuda", stream=None):
        torch = _torch()
        device = torch.device(device)
        if not (device.type == "cuda"):
            _need(False, "checkpoint: must be on a GPU")
        if not (dtype in _TYPES):
            _need(False, "checkpoint: %s is not float32, bfloat16 or float16" % dtype)
        self.shape, self.dtype = tuple(int(n) for n in shape), dtype
        if not (len(self.shape) >= 1 and self.shape[-1] >= 1 and min(self.shape) >= 0):
            _need(False, "checkpoint: the last dimension must be at least 1")
        self.rows, self.width = math.prod(self.shape[:-1]), self.shape[-1]
        groups = self.groups = -(-self.width // KEPT_GROUP)
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        _, other = _stream_of(torch, stream, device)
        with _pool(torch, other):
            self.values = torch.empty(self.rows, groups * KEPT_GROUP, dtype=torch.int8, device=device)
            self.exponents = torch.empty(self.rows, groups, dtype=torch.uint8, device=device)

    def kept(self, what, device) -> Kept:
        torch = _torch()
        values, exponents = self.values, self.exponents
        if not (values.device == device and exponents.device == device):
            _need(False, "%s: the tensors must be on one GPU" % what)
        _packed(what, values, (self.rows, self.groups * KEPT_GROUP), torch.int8, "a checkpoint's values")
        _packed(what, exponents, (self.rows, self.groups), torch.uint8, "a checkpoint's exponents")
        return Kept(values.data_ptr(), exponents.data_ptr())


def _checkpoint_for(torch, what, t, given, other) -> Checkpoint:
    if given is not None:
        if not (isinstance(given, Checkpoint) and given.shape == t.shape and given.dtype == t.dtype):
            _need(False, "%s: a checkpoint of another shape or type" % what)
        return given
    if t.dtype not in _TYPES or not t.dim() or not t.shape[-1]:
        return Checkpoint(t.shape, t.dtype, t.device, other)  # says what is wrong
    c = Checkpoint.__new__(Checkpoint)
    c.shape, c.dtype, device = tuple(t.shape), t.dtype, t.device
    c.width = c.shape[-1]
    c.rows, c.groups = t.numel() // c.width, -(-c.width // KEPT_GROUP)
    with _pool(torch, other):
        c.values = torch.empty((c.rows, c.groups * KEPT_GROUP), dtype=torch.int8, device=device)
        c.exponents = torch.empty((c.rows, c.groups), dtype=torch.uint8, device=device)
    return c


def checkpoint_store(x, checkpoint: Checkpoint | None = None, *, stream=None) -> Checkpoint:
    """mist_kept_store: x (its last dimension contiguous, the others rows at one stride) in 8 bits, into a checkpoint of its shape and
    type or a new one."""
    torch = _torch()
    L = _lib or load()
    what = "checkpoint"
    _no_graph(torch, what, x)
    _here(what, x)
    handle, other = _stream_of(torch, stream, x.device)
    rows, stride = _flat(what, x)
    c = _checkpoint_for(torch, what, x, checkpoint, other)
    k = c.kept(what, x.device)
    d = KeptDesc(rows, c.width, stride, _type(x, what))
    _on_device(torch, x.device, L.mist_kept_store, ctypes.byref(d), x.data_ptr(), k.values, k.exponents, handle)
    if other is not None:
        _used_on(other, x, c.values, c.exponents)
    return c


def checkpoint_load(checkpoint: Checkpoint, *, out=None, dtype=None, stream=None):
    """mist_kept_load: the kept values, in out or a new tensor (of dtype, default the stored tensor's)."""
    torch = _torch()
    L = _lib or load()
    what = "checkpoint"
    device = checkpoint.values.device
    if not (device.type == "cuda"):
        _need(False, "checkpoint: the tensors must be on one GPU")
    handle, other = _stream_of(torch, stream, device)
    if out is None:
        with _pool(torch, other):
            out = torch.empty(checkpoint.shape, dtype=dtype or checkpoint.dtype, device=device)
    if not (tuple(out.shape) == checkpoint.shape and (dtype is None or out.dtype == dtype)):
        _need(False, "%s: out must have the checkpoint's shape" % what)
    if not (out.device == device):
        _need(False, "%s: the tensors must be on one GPU" % what)
    k = checkpoint.kept(what, device)
    rows, stride = _flat(what, out)
    d = KeptDesc(rows, checkpoint.width, stride, _type(out, what))
    _on_device(torch, device, L.mist_kept_load, ctypes.byref(d), k.values, k.exponents, out.data_ptr(), handle)
    if other is not None:
        _used_on(other, checkpoint.values, checkpoint.exponents, out)
    return out


def mlp_act(up, gate=None, *, kind: str = "silu", save=False, out=None, stream=None) -> MlpAct:
    """mist_act_forward: act(gate) * up, or act(up) without a gate (kind 'silu' or 'gelu').  save: True keeps up and gate in 8 bits in new checkpoints,
    a pair (up's, gate's) in these; the result's up and gate are the checkpoints, for mlp_act_grad.  out may be up or gate."""
    torch = _torch()
    L = _lib or load()
    what = "activation"
    _no_graph(torch, what, up, gate)
    _here(what, up, gate, out)
    if not (kind in _ACTS):
        _need(False, "activation: kind must be 'silu' or 'gelu'")
    handle, other = _stream_of(torch, stream, up.device)
    if not (up.dim() >= 1 and up.shape[-1] >= 1):
        _need(False, "activation: the last dimension must be at least 1")
    if not (gate is None or (gate.shape == up.shape and gate.dtype == up.dtype)):
        _need(False, "activation: gate must have up's shape and type")
    if out is None:
        with _pool(torch, other):
            out = _like(torch, up)
    if not (out.shape == up.shape and out.dtype == up.dtype):
        _need(False, "activation: out must have up's shape and type")
    keep = (None, None)
    if save:
        pair = (None, None) if save is True else save
        if not (len(pair) == 2):
            _need(False, "activation: save must be a bool or (up's checkpoint, gate's or None)")
        if gate is None and pair[1] is not None:
            _need(False, "activation: a gate to keep that is not there")
        keep = (_checkpoint_for(torch, what, up, pair[0], other), None if gate is None else _checkpoint_for(torch, what, gate, pair[1], other))
    rows, stride = _flat(what, up)
    d = ActDesc(rows, up.shape[-1], stride, 0 if gate is None else _flat(what, gate)[1], _flat(what, out)[1], 0, _type(up, what), _ACTS[kind])
    k = [None if c is None else ctypes.byref(c.kept(what, up.device)) for c in keep]
    _on_device(torch, up.device, L.mist_act_forward, ctypes.byref(d), up.data_ptr(), _ptr(gate), out.data_ptr(), k[0], k[1], handle)
    if other is not None:
        _used_on(other, up, gate, out, *(t for c in keep if c is not None for t in (c.values, c.exponents)))
    return MlpAct(out, *keep)


def mlp_act_grad(dout, up: Checkpoint, gate: Checkpoint | None = None, *, kind: str = "silu", dup=None, dgate=None, out=None, stream=None):
    """mist_act_backward: (dup, dgate) from the activation's gradient and the kept up and gate.  out, where given, receives the activation
    formed again from them (for the gradient of the projection after it).  dup or dgate may be dout."""
    torch = _torch()
    L = _lib or load()
    what = "activation's gradient"
    _here(what, dout, dup, dgate, out)
    if not (kind in _ACTS):
        _need(False, "activation: kind must be 'silu' or 'gelu'")
    if not (isinstance(up, Checkpoint) and (gate is None or isinstance(gate, Checkpoint))):
        _need(False, "%s: up and gate must be checkpoints" % what)
    if not (up.shape == tuple(dout.shape) and (gate is None or gate.shape == up.shape)):
        _need(False, "%s: a checkpoint of another shape" % what)
    if not (gate is not None or dgate is None):
        _need(False, "%s: of a gate that is not there" % what)
    handle, other = _stream_of(torch, stream, dout.device)
    with _pool(torch, other):
        if dup is None:
            dup = _like(torch, dout)
        if gate is not None and dgate is None:
            dgate = _like(torch, dout)
    for t in (dup, dgate, out):
        if not (t is None or (t.shape == dout.shape and t.dtype == dout.dtype)):
            _need(False, "%s: an output must have dout's shape and type" % what)
    rows, stride = _flat(what, dout)
    d = ActDesc(rows, up.width, _flat(what, dup)[1], 0 if gate is None else _flat(what, dgate)[1], stride, 0 if out is None else _flat(what, out)[1],
                _type(dout, what), _ACTS[kind])
    k = up.kept(what, dout.device), None if gate is None else gate.kept(what, dout.device)
    _on_device(torch, dout.device, L.mist_act_backward, ctypes.byref(d), ctypes.byref(k[0]), None if k[1] is None else ctypes.byref(k[1]),
               dout.data_ptr(), dup.data_ptr(), _ptr(dgate), _ptr(out), handle)
    if other is not None:
        _used_on(other, dout, dup, dgate, out, *(t for c in (up, gate) if c is not None for t in (c.values, c.exponents)))
    return dup, dgate
