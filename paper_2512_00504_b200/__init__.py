"""B200-native G-KV decode-time KV-cache eviction: thin Python binding of the C-ABI library.

The functions here carry the names of the C entry points (``gkv_init``, ``gkv_decode_attn``,
``gkv_evict``, ...) and only marshal arguments: torch tensors become device (or host) pointers,
the current torch stream becomes the ``stream`` argument. Every step of the path runs in the
CUDA kernels of ``libgkv.so``; there is no CPU or PyTorch fallback, and a missing library raises.

``GKVCache`` is a convenience holder that allocates the buffers ``gkv_query_sizes`` asks for with
torch (device memory is all torch is used for) and keeps the context alive.
"""
from __future__ import annotations

import ctypes
import os
import subprocess
from pathlib import Path

_PKG = Path(__file__).resolve().parent
_ROOT = _PKG.parent
# GKV_LIB_VARIANT=check selects the library built with -DGKV_CHECK_BOUNDS (every row index that selection and compaction
# compute is tested before use; see build_library(check_bounds=True)); the default is the production build.
_CHECKED = os.environ.get("GKV_LIB_VARIANT", "") == "check"
LIB_PATH = _PKG / ("libgkv_check.so" if _CHECKED else "libgkv.so")
_SOURCES = ["gkv_api.cu", "gkv_decode.cu", "gkv_evict.cu", "gkv_score.cu", "gkv_score_tc.cu", "gkv_redundancy.cu",
            "gkv_static_scratch.cu", "gkv_store.cu", "gkv_store_attn.cu", "gkv_prefix.cu", "gkv_store_api.cu", "gkv_rotary.cu", "gkv_pages.cu", "gkv_pages_attn.cu", "gkv_pages_stream.cu",
            "gkv_pages_api.cu"]

GKV_OK, GKV_ERR_INVALID_ARG, GKV_ERR_STATE, GKV_ERR_CAPACITY, GKV_ERR_CUDA, GKV_ERR_TIMEOUT, GKV_ERR_UNSUPPORTED, \
    GKV_ERR_SCRATCH_LIMIT, GKV_ERR_INTERNAL = range(9)
GKV_MODE_MAX, GKV_MODE_MEAN, GKV_MODE_SUM, GKV_MODE_LOCAL = range(4)
GKV_STAGE_SCORE, GKV_STAGE_MERGE, GKV_STAGE_SELECT, GKV_STAGE_COMPACT, GKV_STAGE_REDUNDANCY = range(5)
GKV_POLICY_SCORE, GKV_POLICY_STREAMING = range(2)
GKV_STORE_BF16, GKV_STORE_E4M3, GKV_STORE_INT8, GKV_STORE_INT4 = range(4)
GKV_TYPE_BF16, GKV_TYPE_FP16, GKV_TYPE_FP32 = range(3)
GKV_ROTARY_PLAIN, GKV_ROTARY_LINEAR, GKV_ROTARY_NTK, GKV_ROTARY_WAVELENGTH, GKV_ROTARY_YARN = range(5)
ROTARY_SCALINGS = {"plain": GKV_ROTARY_PLAIN, "linear": GKV_ROTARY_LINEAR, "ntk": GKV_ROTARY_NTK, "wavelength": GKV_ROTARY_WAVELENGTH,
                   "yarn": GKV_ROTARY_YARN}
STORE_FORMATS = {"bf16": GKV_STORE_BF16, "e4m3": GKV_STORE_E4M3, "int8": GKV_STORE_INT8, "int4": GKV_STORE_INT4}


class GKVError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {gkv_strerror(status)} (status {status})")


class gkv_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_layers", "batch", "n_q_heads", "n_kv_heads", "head_dim", "budget", "buffer", "window", "interval")] + \
               [("alpha", ctypes.c_float), ("mode", ctypes.c_int32), ("fuse_window_scores", ctypes.c_int32),
                ("track_positions", ctypes.c_int32), ("use_redundancy", ctypes.c_int32),
                ("redundancy_lambda", ctypes.c_float), ("redundancy_threshold", ctypes.c_float),
                ("redundancy_recent", ctypes.c_int32), ("redundancy_eps", ctypes.c_float),
                ("pool_kernel", ctypes.c_int32), ("max_prompt", ctypes.c_int32), ("policy", ctypes.c_int32),
                ("n_sink", ctypes.c_int32)]


class gkv_sizes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in ("k", "v", "f", "sacc", "pos", "len", "workspace", "staging")]


class gkv_buffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "f", "sacc", "pos", "len", "workspace", "staging")]


class gkv_decode_plan_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("grid", "splits", "stages", "ctas_per_sm", "smem_bytes", "tmem_cols")]


class gkv_evict_plan_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("grid", "stages", "ctas_per_sm", "smem_bytes")]


class gkv_score_plan_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tensor_core", "grid", "items", "rows_per_item", "stages", "query_buffers",
                                              "smem_bytes")]


class gkv_store(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("format", "batch", "n_q_heads", "n_kv_heads", "head_dim", "capacity")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class gkv_store_sizes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in ("k", "v", "k_scale", "v_scale")]


class gkv_prefix(ctypes.Structure):
    _fields_ = [("n_prefix", ctypes.c_int32), ("rows", ctypes.c_int32), ("len", ctypes.POINTER(ctypes.c_int32)),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p)]


class gkv_rotary(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("factor", ctypes.c_float),
                ("turns", ctypes.c_void_p)]


class gkv_rotary_rows(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("x_stride", ctypes.c_int64 * 3), ("y_stride", ctypes.c_int64 * 3),
                ("n_heads", ctypes.c_int32)]


class gkv_pages(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("format", "n_q_heads", "n_kv_heads", "head_dim", "n_pages", "page_size", "token_major")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class gkv_page_table(ctypes.Structure):
    _fields_ = [("page", ctypes.c_void_p), ("stride", ctypes.c_int64), ("batch", ctypes.c_int32), ("width", ctypes.c_int32)]


class gkv_memory_model_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in ("full_kv", "compressed_kv", "score_cache")]


def build_library(force: bool = False, verbose: bool = False, check_bounds: bool | None = None) -> Path:
    """Compile csrc/*.cu into libgkv.so for sm_100a with nvcc (cross-compiles without a GPU). check_bounds builds
    libgkv_check.so with -DGKV_CHECK_BOUNDS instead (default: whichever variant this process loads)."""
    check = _CHECKED if check_bounds is None else check_bounds
    out = _PKG / ("libgkv_check.so" if check else "libgkv.so")
    srcs = [_PKG / "csrc" / s for s in _SOURCES if (_PKG / "csrc" / s).exists()]
    deps = srcs + list((_PKG / "csrc").glob("*.h")) + list((_PKG / "csrc").glob("*.cuh")) + [_ROOT / "include" / "gkv.h"]
    if not force and out.exists() and all(out.stat().st_mtime >= d.stat().st_mtime for d in deps):
        return out
    tmp = out.with_suffix(f".so.tmp{os.getpid()}")
    cmd = ["nvcc", "-t", "0", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-shared",
           "-Xcompiler", "-fPIC", "-I", str(_ROOT / "include"), "-o", str(tmp)] + [str(s) for s in srcs]
    if check:
        cmd.insert(1, "-DGKV_CHECK_BOUNDS")
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    subprocess.check_call(cmd)
    os.replace(tmp, out)
    return out


def _binding_built_for() -> str:
    """The torch and Python that csrc/gkv_torch.cpp is compiled against: with others its layouts may not be theirs."""
    import sysconfig

    import torch
    return f"gkv_torch for torch {torch.__version__}, {sysconfig.get_config_var('SOABI')}"


def build_binding(force: bool = False) -> Path:
    """Compile csrc/gkv_torch.cpp (the Python module through which KVStore makes its calls) against this torch."""
    import sysconfig

    import torch
    built_for = _binding_built_for()
    src, out = _PKG / "csrc" / "gkv_torch.cpp", _PKG / "_gkv_torch.so"
    if not force and out.exists() and all(out.stat().st_mtime >= d.stat().st_mtime for d in (src, _ROOT / "include" / "gkv.h")) \
            and built_for.encode() + b"\0" in out.read_bytes():
        return out
    t = Path(torch.__file__).resolve().parent
    cuda = Path(os.environ.get("CUDA_HOME", "/usr/local/cuda"))
    tmp = out.with_suffix(f".so.tmp{os.getpid()}")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                           f'-DGKV_BUILT_FOR="{built_for}"',
                           "-I", str(_ROOT / "include"), "-I", str(t / "include"), "-I", str(t / "include/torch/csrc/api/include"),
                           "-I", str(cuda / "include"), "-I", sysconfig.get_paths()["include"], "-o", str(tmp), str(src),
                           "-L", str(t / "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"])
    os.replace(tmp, out)
    return out


_lib = None
_binding = None


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library. Raises if it has not been built: there is no fallback."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(f"{LIB_PATH} is missing: run __graft_entry__.build() (nvcc, sm_100a) first; "
                               "this package has no CPU or PyTorch fallback")
        L = ctypes.CDLL(str(LIB_PATH))
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        P = ctypes.POINTER
        L.gkv_query_sizes.argtypes = [P(gkv_config), P(gkv_sizes)]
        L.gkv_init.argtypes = [P(vp), P(gkv_config), P(gkv_buffers), vp]
        L.gkv_set_state.argtypes = [vp, i32, i32, i32, i32, i32, vp]
        L.gkv_decode_attn.argtypes = [vp, i32, vp, vp, vp, vp, vp]
        L.gkv_evict.argtypes = [vp, i32, vp, vp, vp]
        L.gkv_evict_stage.argtypes = [vp, i32, i32, vp, vp, vp]
        L.gkv_decode_attn_host.argtypes = [vp, i32, vp, vp, vp, vp, vp]
        L.gkv_evict_host.argtypes = [vp, i32, vp, vp, vp]
        L.gkv_get_state.argtypes = [vp, i32, P(i32), P(i32), P(i32)]
        L.gkv_get_redundancy.argtypes = [vp, i32, vp, vp]
        L.gkv_set_eviction_log.argtypes = [vp, vp]
        L.gkv_compress_prompt.argtypes = [vp, i32, vp, vp, vp, P(i32), vp, vp]
        L.gkv_decode_attn_static.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]
        L.gkv_decode_attn_static.restype = ctypes.c_int
        L.gkv_selftest_bounded_wait.argtypes = [vp, i32, vp]
        L.gkv_selftest_bounded_wait.restype = ctypes.c_int
        L.gkv_launch_count.argtypes = [vp]
        L.gkv_launch_count.restype = i64
        L.gkv_poll_device_status.argtypes = [vp, vp]
        L.gkv_memory_model.argtypes = [P(gkv_config), i64, i32, P(gkv_memory_model_t)]
        L.gkv_decode_launch_plan.argtypes = [P(gkv_config), i32, i32, i32, P(gkv_decode_plan_t)]
        L.gkv_evict_launch_plan.argtypes = [P(gkv_config), i32, i32, P(gkv_evict_plan_t)]
        L.gkv_evict_launch_plan.restype = ctypes.c_int
        L.gkv_score_launch_plan.argtypes = [P(gkv_config), i32, i32, P(gkv_score_plan_t)]
        L.gkv_score_launch_plan.restype = ctypes.c_int
        u64 = ctypes.c_uint64
        L.gkv_store_query_sizes.argtypes = [P(gkv_store), P(gkv_store_sizes)]
        L.gkv_store_write.argtypes = [P(gkv_store), vp, vp, i64, i64, i64, vp, vp, i32, vp]
        L.gkv_store_read.argtypes = [P(gkv_store), vp, vp, i64, i64, i64, vp, vp, i32, vp]
        L.gkv_store_attn_workspace.argtypes = [P(gkv_store), i32, i32, P(u64)]
        L.gkv_store_attn.argtypes = [P(gkv_store), vp, i32, vp, vp, vp, P(gkv_prefix), vp, vp, vp, u64, vp]
        L.gkv_decode_attn_prefix.argtypes = [vp, i32, vp, vp, vp, P(gkv_prefix), vp, vp, u64, vp]
        L.gkv_selftest_prefix_wait.argtypes = [vp]
        f64 = ctypes.c_double
        L.gkv_rotary_frequencies.argtypes = [f64, i32, i32, f64, f64, f64, f64, P(f64), P(ctypes.c_float)]
        L.gkv_rotary_turns.argtypes = [P(f64), i32, P(u64)]
        L.gkv_rotary_apply.argtypes = [P(gkv_rotary), i32, i32, i32, vp, i64, i64, vp, P(gkv_rotary_rows), P(gkv_rotary_rows), i32, vp]
        L.gkv_pages_query_sizes.argtypes = [P(gkv_pages), P(gkv_store_sizes)]
        L.gkv_pages_append.argtypes = [P(gkv_pages), P(gkv_page_table), vp, vp, i64, i64, i64, vp, vp, i32, P(gkv_rotary), vp, i64, i64, vp]
        L.gkv_pages_read.argtypes = [P(gkv_pages), P(gkv_page_table), vp, vp, i64, i64, i64, vp, vp, i32, vp]
        L.gkv_pages_attn_workspace.argtypes = [P(gkv_pages), i32, P(u64)]
        L.gkv_pages_attn.argtypes = [P(gkv_pages), P(gkv_page_table), vp, i32, vp, i64, vp, vp, i64, P(gkv_rotary), vp, vp, vp, vp, u64, vp]
        L.gkv_selftest_pages_wait.argtypes = [i32] + L.gkv_pages_attn.argtypes
        for name in ("gkv_rotary_frequencies", "gkv_rotary_turns", "gkv_rotary_apply", "gkv_pages_query_sizes", "gkv_pages_append",
                     "gkv_pages_read", "gkv_pages_attn_workspace", "gkv_pages_attn", "gkv_selftest_pages_wait"):
            getattr(L, name).restype = ctypes.c_int
        for name in ("gkv_store_query_sizes", "gkv_store_write", "gkv_store_read", "gkv_store_attn_workspace",
                     "gkv_store_attn", "gkv_decode_attn_prefix", "gkv_selftest_prefix_wait"):
            getattr(L, name).restype = ctypes.c_int
        L.gkv_strerror.argtypes = [ctypes.c_int]
        L.gkv_strerror.restype = ctypes.c_char_p
        L.gkv_destroy.argtypes = [vp]
        L.gkv_destroy.restype = None
        for name in ("gkv_query_sizes", "gkv_init", "gkv_set_state", "gkv_decode_attn", "gkv_evict", "gkv_evict_stage",
                     "gkv_decode_attn_host", "gkv_evict_host", "gkv_get_state", "gkv_get_redundancy", "gkv_set_eviction_log", "gkv_compress_prompt", "gkv_poll_device_status",
                     "gkv_memory_model", "gkv_decode_launch_plan"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _torch_binding():
    """The module that takes torch tensors to the store calls, bound to the loaded library. Raises if it has not been built."""
    global _binding
    if _binding is None:
        import importlib.util

        import torch  # noqa: F401  (its libraries have to be loaded first)
        path = _PKG / "_gkv_torch.so"
        if not path.exists():
            raise RuntimeError(f"{path} is missing: run __graft_entry__.build() first")
        spec = importlib.util.spec_from_file_location("_gkv_torch", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        if module.built_for != _binding_built_for():
            raise RuntimeError(f"{path} is a {module.built_for}, this is {_binding_built_for()}: run __graft_entry__.build() again")
        L = lib()
        module.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
            L.gkv_store_write, L.gkv_store_read, L.gkv_store_attn, L.gkv_pages_append, L.gkv_pages_read, L.gkv_pages_attn, L.gkv_rotary_apply)))
        _binding = module
    return _binding


def _check(status: int, what: str) -> None:
    if status != GKV_OK:
        raise GKVError(status, what)


def _ptr(t):
    """Pointer of a torch tensor (device or host), a raw int, or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return ctypes.c_void_p(t)
    assert t.is_contiguous()
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def make_config(*, n_layers, batch, h_q, h_kv, d=128, b, buffer, w, s, alpha=0.8, mode=GKV_MODE_MAX,
                fuse_window_scores=True, track_positions=False, redundancy_lambda=None, redundancy_threshold=0.5,
                redundancy_recent=None, redundancy_eps=1e-6, pool_kernel=0, max_prompt=0, policy=GKV_POLICY_SCORE, n_sink=0,
                **_ignored) -> gkv_config:
    """redundancy_lambda=None leaves the redundancy term off; redundancy_recent defaults to the window."""
    use = redundancy_lambda is not None
    return gkv_config(n_layers, batch, h_q, h_kv, d, b, buffer, w, s, alpha, mode,
                      int(fuse_window_scores), int(track_positions), int(use), float(redundancy_lambda if use else 1.0),
                      float(redundancy_threshold), int(w if redundancy_recent is None else redundancy_recent),
                      float(redundancy_eps), int(pool_kernel), int(max_prompt), int(policy), int(n_sink))


# ------------------------------------------------------------------ C-ABI calls, same names
def gkv_strerror(status: int) -> str:
    return lib().gkv_strerror(int(status)).decode()


def gkv_query_sizes(cfg: gkv_config) -> gkv_sizes:
    out = gkv_sizes()
    _check(lib().gkv_query_sizes(ctypes.byref(cfg), ctypes.byref(out)), "gkv_query_sizes")
    return out


def gkv_decode_launch_plan(cfg: gkv_config, n_layers_in_launch: int, window_step: bool = False, sm_count: int = 148) -> gkv_decode_plan_t:
    out = gkv_decode_plan_t()
    _check(lib().gkv_decode_launch_plan(ctypes.byref(cfg), int(n_layers_in_launch), int(bool(window_step)), int(sm_count),
                                        ctypes.byref(out)), "gkv_decode_launch_plan")
    return out


def gkv_score_launch_plan(cfg: gkv_config, n_layers_in_launch: int, sm_count: int = 148) -> gkv_score_plan_t:
    out = gkv_score_plan_t()
    _check(lib().gkv_score_launch_plan(ctypes.byref(cfg), int(n_layers_in_launch), int(sm_count), ctypes.byref(out)),
           "gkv_score_launch_plan")
    return out


def gkv_evict_launch_plan(cfg: gkv_config, n_layers_in_launch: int, sm_count: int = 148) -> gkv_evict_plan_t:
    out = gkv_evict_plan_t()
    _check(lib().gkv_evict_launch_plan(ctypes.byref(cfg), int(n_layers_in_launch), int(sm_count), ctypes.byref(out)),
           "gkv_evict_launch_plan")
    return out


def gkv_memory_model(cfg: gkv_config, seq_len: int, elem_bytes: int = 2) -> gkv_memory_model_t:
    out = gkv_memory_model_t()
    _check(lib().gkv_memory_model(ctypes.byref(cfg), int(seq_len), int(elem_bytes), ctypes.byref(out)), "gkv_memory_model")
    return out


def gkv_init(cfg: gkv_config, buffers: gkv_buffers) -> ctypes.c_void_p:
    ctx = ctypes.c_void_p()
    _check(lib().gkv_init(ctypes.byref(ctx), ctypes.byref(cfg), ctypes.byref(buffers), _stream()), "gkv_init")
    return ctx


def gkv_set_state(ctx, layer, length, n_hist, since_evict, window_scores_valid=False):
    _check(lib().gkv_set_state(ctx, layer, length, n_hist, since_evict, int(window_scores_valid), _stream()), "gkv_set_state")


def gkv_decode_attn(ctx, layer, q, k_new, v_new, out):
    _check(lib().gkv_decode_attn(ctx, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _stream()), "gkv_decode_attn")


def gkv_evict(ctx, layer, q_window=None, kept_idx_out=None):
    _check(lib().gkv_evict(ctx, layer, _ptr(q_window), _ptr(kept_idx_out), _stream()), "gkv_evict")


def gkv_evict_stage(ctx, layer, stage, q_window=None, kept_idx_out=None):
    _check(lib().gkv_evict_stage(ctx, layer, stage, _ptr(q_window), _ptr(kept_idx_out), _stream()), "gkv_evict_stage")


def gkv_decode_attn_host(ctx, layer, q, k_new, v_new, out):
    _check(lib().gkv_decode_attn_host(ctx, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _stream()),
           "gkv_decode_attn_host")


def gkv_evict_host(ctx, layer, q_window=None, kept_idx_out=None):
    _check(lib().gkv_evict_host(ctx, layer, _ptr(q_window), _ptr(kept_idx_out), _stream()), "gkv_evict_host")


def gkv_decode_attn_static(q, k_new, v_new, k_cache, v_cache, out, length):
    """Workspace-free decode step for one layer (see gkv.h): for callers that cannot allocate device
    memory when they call. k_cache / v_cache are [batch][h_kv][capacity][128]; `length` is the number of
    rows already in the cache; the new row is written at that index. Calls must not overlap on the GPU."""
    batch, h_q, _ = q.shape
    _, h_kv, capacity, _ = k_cache.shape
    _check(lib().gkv_decode_attn_static(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(out),
                                        batch, h_q, h_kv, capacity, int(length), _stream()), "gkv_decode_attn_static")


def gkv_get_state(ctx, layer):
    a, b, c = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(lib().gkv_get_state(ctx, layer, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)), "gkv_get_state")
    return a.value, b.value, c.value


def gkv_compress_prompt(ctx, layer, k_prompt, v_prompt, q_window, prompt_len, kept_idx_out=None):
    """prompt_len: sequence of batch ints (host)."""
    lens = (ctypes.c_int32 * len(prompt_len))(*[int(x) for x in prompt_len])
    _check(lib().gkv_compress_prompt(ctx, layer, _ptr(k_prompt), _ptr(v_prompt), _ptr(q_window), lens,
                                     _ptr(kept_idx_out), _stream()), "gkv_compress_prompt")


def gkv_set_eviction_log(ctx, log):
    _check(lib().gkv_set_eviction_log(ctx, _ptr(log)), "gkv_set_eviction_log")


def gkv_get_redundancy(ctx, layer, out):
    _check(lib().gkv_get_redundancy(ctx, layer, _ptr(out), _stream()), "gkv_get_redundancy")


def gkv_launch_count(ctx) -> int:
    return int(lib().gkv_launch_count(ctx))


def gkv_poll_device_status(ctx):
    _check(lib().gkv_poll_device_status(ctx, _stream()), "gkv_poll_device_status")


def gkv_selftest_bounded_wait(ctx, spins: int = 1024):
    _check(lib().gkv_selftest_bounded_wait(ctx, int(spins), _stream()), "gkv_selftest_bounded_wait")


def gkv_destroy(ctx):
    lib().gkv_destroy(ctx)


# The calls on a store that take tensors are made by KVStore (below), through csrc/gkv_torch.cpp.
def gkv_store_query_sizes(store: gkv_store) -> gkv_store_sizes:
    out = gkv_store_sizes()
    _check(lib().gkv_store_query_sizes(ctypes.byref(store), ctypes.byref(out)), "gkv_store_query_sizes")
    return out


def gkv_store_attn_workspace(store: gkv_store, n_prefix: int = 0, prefix_rows: int = 0) -> int:
    out = ctypes.c_uint64()
    _check(lib().gkv_store_attn_workspace(ctypes.byref(store), int(n_prefix), int(prefix_rows), ctypes.byref(out)),
           "gkv_store_attn_workspace")
    return out.value


def gkv_decode_attn_prefix(ctx, layer, q, k_new, v_new, prefix, out, workspace):
    """prefix: a Prefix with the context's KV heads (a context does not say how many: GKVCache.decode_attn_prefix checks);
    workspace: a uint8 tensor of gkv_store_attn_workspace bytes (GKVCache.prefix_workspace)."""
    _check(lib().gkv_decode_attn_prefix(ctx, layer, _ptr(q), _ptr(k_new), _ptr(v_new), ctypes.byref(prefix.desc), _ptr(out),
                                        _ptr(workspace), workspace.numel(), _stream()), "gkv_decode_attn_prefix")


def gkv_selftest_prefix_wait(ctx):
    _check(lib().gkv_selftest_prefix_wait(ctx), "gkv_selftest_prefix_wait")


# The calls that rotate tensors and take pages are made by Rotary and PagedStore (below), through csrc/gkv_torch.cpp.
def gkv_rotary_frequencies(theta, rot_dim, scaling=GKV_ROTARY_PLAIN, scale=1.0, original=0.0, low=0.0, high=0.0):
    """(radians a position of the rot_dim / 2 pairs, factor); the scalings' formulas are in gkv.h."""
    out, factor = (ctypes.c_double * max(1, int(rot_dim) // 2))(), ctypes.c_float()
    _check(lib().gkv_rotary_frequencies(float(theta), _int32(rot_dim, "rot_dim"), int(scaling), float(scale), float(original), float(low),
                                        float(high), out, ctypes.byref(factor)), "gkv_rotary_frequencies")
    return list(out), factor.value


def gkv_rotary_turns(radians):
    """Frequencies in radians a position as units of 2^-64 turns."""
    radians = [float(f) for f in radians]
    out = (ctypes.c_uint64 * max(1, len(radians)))()
    _check(lib().gkv_rotary_turns((ctypes.c_double * max(1, len(radians)))(*radians), len(radians), out), "gkv_rotary_turns")
    return list(out[:len(radians)])


def gkv_pages_query_sizes(pages: gkv_pages) -> gkv_store_sizes:
    out = gkv_store_sizes()
    _check(lib().gkv_pages_query_sizes(ctypes.byref(pages), ctypes.byref(out)), "gkv_pages_query_sizes")
    return out


def gkv_pages_attn_workspace(pages: gkv_pages, batch: int) -> int:
    out = ctypes.c_uint64()
    _check(lib().gkv_pages_attn_workspace(ctypes.byref(pages), _int32(batch, "batch"), ctypes.byref(out)), "gkv_pages_attn_workspace")
    return out.value


def gkv_selftest_pages_wait(store: "PagedStore", step, table, length, q, out, k_new=None, v_new=None, lse=None, max_len=0):
    """PagedStore.attn without a rotation, whose warps take every wait from their step `step` on for expired. All tensors contiguous."""
    import torch
    dev, batch, bf16 = store.device, table.shape[0], torch.bfloat16
    t = gkv_page_table(_tensor(table, "table", torch.int32, table.shape, dev), table.shape[1], batch, table.shape[1])
    new = [None if x is None else _tensor(x, n, bf16, (batch, store.h_kv, 128), dev) for x, n in ((k_new, "k_new"), (v_new, "v_new"))]
    _check(lib().gkv_selftest_pages_wait(
        _int32(step, "step"), ctypes.byref(store.desc), ctypes.byref(t), _tensor(length, "length", torch.int32, (batch,), dev),
        _int32(max_len, "max_len"), _tensor(q, "q", bf16, (batch, store.h_q, 128), dev), store.h_q * 128, *new, store.h_kv * 128, None, None,
        _tensor(out, "out", bf16, (batch, store.h_q, 128), dev), None if lse is None else _tensor(lse, "lse", torch.float32, (batch, store.h_q), dev),
        *store._ws, torch.cuda.current_stream(dev).cuda_stream), "gkv_selftest_pages_wait")


# ------------------------------------------------------------------ buffer holder
class GKVCache:
    """Allocates the caller-owned buffers with torch and owns the context."""

    def __init__(self, cfg: gkv_config, device="cuda:0", staging: bool = False):
        import torch
        self.cfg = cfg
        self.device = torch.device(device)
        self.sizes = gkv_query_sizes(cfg)
        L, B, H, C = cfg.n_layers, cfg.batch, cfg.n_kv_heads, cfg.budget + cfg.buffer
        self.C = C
        with torch.cuda.device(self.device):
            dev = self.device
            self.k = torch.empty((L, B, H, C, cfg.head_dim), dtype=torch.bfloat16, device=dev)
            self.v = torch.empty_like(self.k)
            self.f = torch.empty((L, B, H, C), dtype=torch.float32, device=dev)
            self.sacc = torch.empty_like(self.f)
            self.pos = torch.empty((L, B, H, C), dtype=torch.int32, device=dev) if cfg.track_positions else None
            self.len = torch.empty((2, L, B), dtype=torch.int32, device=dev)
            self.workspace = torch.empty(int(self.sizes.workspace), dtype=torch.uint8, device=dev)
            self.staging = torch.empty(int(self.sizes.staging), dtype=torch.uint8, device=dev) if staging else None
            assert self.k.numel() * 2 == self.sizes.k and self.f.numel() * 4 == self.sizes.f
            bufs = gkv_buffers(self.k.data_ptr(), self.v.data_ptr(), self.f.data_ptr(), self.sacc.data_ptr(),
                               self.pos.data_ptr() if self.pos is not None else None, self.len.data_ptr(),
                               self.workspace.data_ptr(), self.staging.data_ptr() if staging else None)
            self.ctx = gkv_init(cfg, bufs)

    def close(self):
        if getattr(self, "ctx", None) is not None:
            gkv_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # thin forwards
    def set_state(self, layer, length, n_hist, since_evict, window_scores_valid=False):
        gkv_set_state(self.ctx, layer, length, n_hist, since_evict, window_scores_valid)

    def decode_attn(self, layer, q, k_new, v_new, out):
        gkv_decode_attn(self.ctx, layer, q, k_new, v_new, out)

    def evict(self, layer, q_window=None, kept_idx_out=None):
        gkv_evict(self.ctx, layer, q_window, kept_idx_out)

    def evict_stage(self, layer, stage, q_window=None, kept_idx_out=None):
        gkv_evict_stage(self.ctx, layer, stage, q_window, kept_idx_out)

    def state(self, layer=0):
        return gkv_get_state(self.ctx, layer)

    def compress_prompt(self, layer, k_prompt, v_prompt, q_window, prompt_len, kept_idx_out=None):
        gkv_compress_prompt(self.ctx, layer, k_prompt, v_prompt, q_window, prompt_len, kept_idx_out)

    def enable_eviction_log(self):
        """Allocates [n_layers][batch][h_kv][buffer] int32 and has every eviction write its evicted tokens there."""
        import torch
        cfg = self.cfg
        self.evict_log = torch.full((cfg.n_layers, cfg.batch, cfg.n_kv_heads, cfg.buffer), -1, dtype=torch.int32,
                                    device=self.device)
        gkv_set_eviction_log(self.ctx, self.evict_log)
        return self.evict_log

    def redundancy(self, layer=0):
        """cbar [batch][h_kv][C] of the last eviction of `layer` (redundancy term on)."""
        import torch
        out = torch.empty((self.cfg.batch, self.cfg.n_kv_heads, self.C), dtype=torch.float32, device=self.device)
        gkv_get_redundancy(self.ctx, layer, out)
        return out

    def prefix_workspace(self, n_prefix, prefix_rows):
        """Workspace of decode_attn_prefix for up to n_prefix prefixes of up to prefix_rows rows."""
        import torch
        c, n_prefix, prefix_rows = self.cfg, _int32(n_prefix, "n_prefix"), _int32(prefix_rows, "prefix_rows")
        shape = gkv_store(GKV_STORE_BF16, c.batch, c.n_q_heads, c.n_kv_heads, c.head_dim, self.C)
        return torch.empty(gkv_store_attn_workspace(shape, n_prefix, prefix_rows), dtype=torch.uint8, device=self.device)

    def decode_attn_prefix(self, layer, q, k_new, v_new, prefix, out, workspace):
        _fitting(prefix, self.cfg.n_kv_heads, self.k.device, "cache")
        gkv_decode_attn_prefix(self.ctx, layer, q, k_new, v_new, prefix, out, workspace)

    def poll(self):
        gkv_poll_device_status(self.ctx)


def _tensor(t, what, dtype, shape, device):
    """Data pointer of a contiguous tensor of this type, shape and device."""
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} on {device} is needed, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}" + ("" if t.is_contiguous() else ", not contiguous"))
    return t.data_ptr()


def _int32(n, what):
    """n as an int that the C calls' 32-bit arguments hold (ctypes cuts the rest off without a word)."""
    n = int(n)
    if not -2 ** 31 <= n < 2 ** 31:
        raise ValueError(f"{what} {n} does not fit 32 bits")
    return n


def _fitting(prefix, h_kv, device, what):
    """The C calls take the head count of a prefix's rows from the store or the context: others would be read out of place."""
    if prefix.h_kv != h_kv or prefix.k.device != device:
        raise ValueError(f"the prefix has {prefix.h_kv} KV heads on {prefix.k.device}, the {what} {h_kv} on {device}")


class Prefix:
    """Rows that the sequences of a batch share: k, v [n_prefix][kv heads][rows][128] bf16 on the device, of which prefix p
    has its first lengths[p] in use. Sequence i of a batch belongs to prefix i // (batch // n_prefix)."""

    def __init__(self, k, v, lengths):
        import torch
        if k.dim() != 4 or k.shape[3] != 128 or k.device.type != "cuda":
            raise ValueError("k, v: bf16 device tensors [n_prefix][kv heads][rows][128]")
        pk, pv = (_tensor(t, n, torch.bfloat16, k.shape, k.device) for t, n in ((k, "k"), (v, "v")))
        lengths = [_int32(n, "length") for n in lengths]
        if len(lengths) != k.shape[0]:
            raise ValueError(f"{len(lengths)} lengths for {k.shape[0]} prefixes")
        self.k, self.v, self.h_kv = k, v, k.shape[1]
        self._len = (ctypes.c_int32 * len(lengths))(*lengths)
        self.desc = gkv_prefix(k.shape[0], k.shape[2], self._len, pk, pv)
        self.at = ctypes.addressof(self.desc)


class KVStore:
    """K and V rows of one layer in 16, 8 or 4 bits (layouts in gkv.h), with the workspace of its attention.

    fmt: "bf16", "e4m3", "int8" or "int4". The buffers are allocated here (uninitialised: rows are written before they are
    read) or given: (k, v, k_scale, v_scale), for bf16 (k, v). max_prefix and n_prefix: the longest prefix and the most
    prefixes that attn will be given. Calls of one store must not overlap on the GPU (they share the workspace). What has been
    allocated here may be dropped while streams still work on it (given buffers and a call's tensors are the caller's to keep)."""

    def __init__(self, fmt, *, batch, h_q, h_kv, capacity, device=None, buffers=None, max_prefix=0, n_prefix=0):
        import torch
        self.fmt, self.batch, self.h_q, self.h_kv, self.capacity = fmt, batch, h_q, h_kv, capacity
        if fmt not in STORE_FORMATS:
            raise ValueError(f"format {fmt!r}: one of {sorted(STORE_FORMATS)} is needed")
        for n, what in ((batch, "batch"), (h_q, "h_q"), (h_kv, "h_kv"), (capacity, "capacity"), (n_prefix, "n_prefix"), (max_prefix, "max_prefix")):
            _int32(n, what)
        self.desc = gkv_store(STORE_FORMATS[fmt], batch, h_q, h_kv, 128, capacity)
        self.sizes = gkv_store_query_sizes(self.desc)
        given = buffers is not None
        code = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8, "int4": torch.uint8}[fmt]
        scales = {"bf16": 0, "e4m3": 1, "int8": 1, "int4": 4}[fmt]
        shape, s_shape = torch.Size((batch, h_kv, capacity, 64 if fmt == "int4" else 128)), torch.Size((batch, h_kv, capacity, scales))
        if buffers is None:
            device = torch.device(device or "cuda")
            buffers = [torch.empty(shape, dtype=code, device=device) for _ in range(2)]
            if scales:
                buffers += [torch.empty(s_shape, dtype=torch.bfloat16, device=device) for _ in range(2)]
        if len(buffers) != (4 if scales else 2):
            raise ValueError(f"{len(buffers)} buffers for format {fmt}")
        self.device = buffers[0].device
        for t, n in zip(buffers, ("k", "v")):
            setattr(self.desc, n, _tensor(t, n, code, shape, self.device))
        for t, n in zip(buffers[2:], ("k_scale", "v_scale")):
            setattr(self.desc, n, _tensor(t, n, torch.bfloat16, s_shape, self.device))
        self.k, self.v = buffers[0], buffers[1]
        self.k_scale, self.v_scale = (buffers[2], buffers[3]) if scales else (None, None)
        self.workspace = torch.empty(gkv_store_attn_workspace(self.desc, n_prefix, max_prefix), dtype=torch.uint8, device=self.device)
        if self.device.type != "cuda":
            raise ValueError(f"the buffers are on {self.device}")
        self._call = _torch_binding()
        # what has been allocated here, and on which stream
        self._held = (torch.cuda.current_stream(self.device).cuda_stream, self.device.index, self.workspace) + (() if given else tuple(buffers))
        self._at = (ctypes.addressof(self.desc), self.device.index)
        self._ws = (self.workspace.data_ptr(), self.workspace.numel())

    def write(self, k, v, first=None, count=None):
        """Quantise tokens into rows first[i] .. first[i] + count[i] - 1 of every sequence i. k, v: bf16 [batch][tokens][kv
        heads][128] with any strides whose last one is 1, the same ones for both; first, count: int32 on the device (None: 0
        and all tokens)."""
        at, dev = self._at
        _check(self._call.copy(False, at, dev, k, v, first, count), "gkv_store_write")
        self._call.in_use(self._held)

    def read(self, k, v, first=None, count=None):
        """Read the same rows back as bf16 into k and v, whose rows may not overlap; tokens from count[i] on are left as they were."""
        at, dev = self._at
        _check(self._call.copy(True, at, dev, k, v, first, count), "gkv_store_read")
        self._call.in_use(self._held)

    def attn(self, length, q, out, k_new=None, v_new=None, prefix=None, lse=None, max_len=0):
        """Decode attention over rows 0 .. length[i] - 1 (int32 on the device), the new token (appended at row length[i]) and
        the sequence's prefix. The caller counts length up. max_len: the longest length (0: the capacity)."""
        at, dev = self._at
        ws, ws_bytes = self._ws
        pre = 0
        if prefix is not None:
            _fitting(prefix, self.h_kv, self.device, "store")
            pre = prefix.at
        _check(self._call.attn(at, dev, length, max_len, q, k_new, v_new, pre, out, lse, ws, ws_bytes), "gkv_store_attn")
        self._call.in_use(self._held)


class Rotary:
    """Rotary positions: the frequencies of the pairs of a head's first 2 len(frequencies) elements, in radians a position, and how the
    pairs lie (formulas in gkv.h). Rotary.scaled makes the usual ones."""

    def __init__(self, frequencies, *, head_dim=128, interleaved=False, factor=1.0, device=None):
        import numpy as np
        import torch
        turns = np.array(gkv_rotary_turns(frequencies), np.uint64)
        head_dim, rot_dim = _int32(head_dim, "head_dim"), 2 * len(turns)
        if not 2 <= rot_dim <= head_dim or head_dim % 2 or head_dim > 512 or not abs(float(factor)) < float("inf"):
            raise ValueError(f"{len(turns)} frequencies, factor {factor}: 1 to head_dim / 2 of them and a finite factor are needed, with an even "
                             f"head_dim of 2 to 512 ({head_dim})")
        device = torch.device(device or "cuda")
        if device.type != "cuda":
            raise ValueError(f"the frequencies would be on {device}")
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        self.device, self.head_dim, self.rot_dim = self.turns.device, head_dim, rot_dim
        self.desc = gkv_rotary(head_dim, rot_dim, int(bool(interleaved)), float(factor), self.turns.data_ptr())
        self.at = ctypes.addressof(self.desc)
        self._call = _torch_binding()
        self._held = (torch.cuda.current_stream(self.device).cuda_stream, self.device.index, self.turns)

    @classmethod
    def scaled(cls, theta, rot_dim=128, *, scaling="plain", scale=1.0, original=0.0, low=1.0, high=None, head_dim=128, interleaved=False,
               device=None):
        """Base frequencies theta^(-2i / rot_dim), for a context `scale` times the original one by one of ROTARY_SCALINGS. low, high: the
        turns in the original context between which "wavelength" (high: 4 by default) and "yarn" (32) blend."""
        if scaling not in ROTARY_SCALINGS:
            raise ValueError(f"scaling {scaling!r}: one of {sorted(ROTARY_SCALINGS)} is needed")
        high = (4.0 if scaling == "wavelength" else 32.0) if high is None else high
        frequencies, factor = gkv_rotary_frequencies(theta, rot_dim, ROTARY_SCALINGS[scaling], scale, original, low, high)
        return cls(frequencies, head_dim=head_dim, interleaved=interleaved, factor=factor, device=device)

    def apply(self, pos, q, k=None, *, q_out=None, k_out=None, count=None, transpose=False):
        """Rotate q and k in one launch, in place or into q_out, k_out. q, k: [batch][tokens][their heads][head_dim] in bf16, fp16 or fp32, any
        strides whose last one is 1; pos: int32 [batch][tokens] on the device; count: int32 [batch], tokens from count[i] on are left as
        they were. transpose turns the other way: given the gradients of what was rotated, it leaves those of q and k. Nothing is recorded for a
        backward pass: tensors that require grad are refused unless gradients are off (torch.no_grad(), or within a torch.autograd.Function,
        whose backward is the same call with transpose)."""
        _check(self._call.rotary(self.at, self.device.index, pos, q, k, q_out, k_out, count, transpose), "gkv_rotary_apply")
        self._call.in_use(self._held)


class PagedStore:
    """K and V rows of one layer in pages (layouts in gkv.h), with the workspace of their attention for up to max_batch sequences.

    fmt: "bf16", "e4m3", "int8" or "int4". The pages are allocated here (uninitialised) or given as buffers: (k, v, k_scale, v_scale),
    for bf16 (k, v), each [pages][h_kv][page_size][...] or, token_major, [pages][page_size][h_kv][...]. Every call takes the table of its
    sequences, int32 [batch][places] on the device: row r of sequence i is row r % page_size of page table[i][r // page_size]. Calls of
    one store must not overlap on the GPU (they share the workspace); the stores of a model's layers may share one (workspace: another
    store's, 22 MB) if theirs do not either. What has been allocated here may be dropped while streams still work on it (given buffers, a given
    workspace and a call's tensors are the caller's to keep)."""

    def __init__(self, fmt, *, pages, page_size, h_q, h_kv, max_batch, token_major=False, device=None, buffers=None, workspace=None):
        import torch
        if fmt not in STORE_FORMATS:
            raise ValueError(f"format {fmt!r}: one of {sorted(STORE_FORMATS)} is needed")
        pages, page_size, h_q, h_kv, max_batch = (_int32(n, what) for n, what in (
            (pages, "pages"), (page_size, "page_size"), (h_q, "h_q"), (h_kv, "h_kv"), (max_batch, "max_batch")))
        self.fmt, self.pages, self.page_size, self.h_q, self.h_kv, self.max_batch = fmt, pages, page_size, h_q, h_kv, max_batch
        self.token_major = bool(token_major)
        self.desc = gkv_pages(STORE_FORMATS[fmt], h_q, h_kv, 128, pages, page_size, int(self.token_major))
        self.sizes = gkv_pages_query_sizes(self.desc)
        given = buffers is not None
        code = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8, "int4": torch.uint8}[fmt]
        scales = {"bf16": 0, "e4m3": 1, "int8": 1, "int4": 4}[fmt]
        rows = (pages, page_size, h_kv) if self.token_major else (pages, h_kv, page_size)
        shape, s_shape = torch.Size((*rows, 64 if fmt == "int4" else 128)), torch.Size((*rows, scales))
        ws_bytes = gkv_pages_attn_workspace(self.desc, max_batch)
        if buffers is None:
            device = torch.device(device or "cuda")
            buffers = [torch.empty(shape, dtype=code, device=device) for _ in range(2)]
            if scales:
                buffers += [torch.empty(s_shape, dtype=torch.bfloat16, device=device) for _ in range(2)]
        if len(buffers) != (4 if scales else 2):
            raise ValueError(f"{len(buffers)} buffers for format {fmt}")
        self.device = buffers[0].device
        for t, n in zip(buffers, ("k", "v")):
            setattr(self.desc, n, _tensor(t, n, code, shape, self.device))
        for t, n in zip(buffers[2:], ("k_scale", "v_scale")):
            setattr(self.desc, n, _tensor(t, n, torch.bfloat16, s_shape, self.device))
        self.k, self.v = buffers[0], buffers[1]
        self.k_scale, self.v_scale = (buffers[2], buffers[3]) if scales else (None, None)
        if self.device.type != "cuda":
            raise ValueError(f"the buffers are on {self.device}")
        if workspace is not None and (workspace.dtype != torch.uint8 or workspace.device != self.device or not workspace.is_contiguous()
                                      or workspace.numel() < ws_bytes):
            raise ValueError(f"workspace: {ws_bytes} contiguous bytes (uint8) on {self.device} are needed")
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device) if workspace is None else workspace
        self._call = _torch_binding()
        # what has been allocated here, and on which stream
        self._held = (torch.cuda.current_stream(self.device).cuda_stream, self.device.index) + (() if given else tuple(buffers)) + \
            ((self.workspace,) if workspace is None else ())
        self._at = (ctypes.addressof(self.desc), self.device.index, max_batch)
        self._ws = (self.workspace.data_ptr(), self.workspace.numel())

    def _rotary(self, rotary):
        if rotary is None:
            return 0
        if rotary.head_dim != 128 or rotary.device != self.device:
            raise ValueError(f"the rotary is for heads of {rotary.head_dim} on {rotary.device}, the pages hold 128 on {self.device}")
        return rotary.at

    def _used(self, rotary):
        self._call.in_use(self._held)
        if rotary is not None:
            self._call.in_use(rotary._held)

    def append(self, table, k, v, first=None, count=None, rotary=None, pos=None):
        """Quantise tokens into rows first[i] .. first[i] + count[i] - 1 of every sequence i, keys rotated on the way if there is a rotary, at
        positions pos (int32 [batch][tokens] on the device; None: the rows' numbers). k, v: bf16 [batch][tokens][kv heads][128] with any
        strides whose last one is 1, the same ones for both; first, count: int32 on the device (None: 0 and all tokens)."""
        at, dev, _ = self._at
        _check(self._call.pages_copy(False, at, dev, table, k, v, first, count, self._rotary(rotary), pos), "gkv_pages_append")
        self._used(rotary)

    def read(self, table, k, v, first=None, count=None):
        """Read the same rows back as bf16 into k and v, whose rows may not overlap; tokens from count[i] on are left as they were."""
        at, dev, _ = self._at
        _check(self._call.pages_copy(True, at, dev, table, k, v, first, count, 0, None), "gkv_pages_read")
        self._used(None)

    def attn(self, table, length, q, out, k_new=None, v_new=None, rotary=None, pos=None, lse=None, max_len=0):
        """Decode attention over rows 0 .. length[i] - 1 (int32 on the device) and the new token, which is appended at row length[i]. With a
        rotary, q and k_new are rotated on the way, at pos[i] (int32 on the device; None: the number of the last row). q, k_new, v_new:
        bf16 [batch][their heads][128], slices of one projection's output if need be. The caller counts length up. max_len: the longest
        length (0: what the table can hold)."""
        at, dev, most = self._at
        ws, ws_bytes = self._ws
        _check(self._call.pages_attn(at, dev, most, table, length, max_len, q, k_new, v_new, self._rotary(rotary), pos, out, lse, ws, ws_bytes),
               "gkv_pages_attn")
        self._used(rotary)
