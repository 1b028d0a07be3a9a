"""Builds liblayoutcopy.so (host algebra + planners + gfx950 kernels) in-tree with hipcc."""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB_PATH = os.path.join(HERE, "liblayoutcopy.so")
OBJ_DIR = os.path.join(HERE, "_build")
SOURCES = ["layout.cpp", "algebra.cpp", "semimodule.cpp", "plan.cpp", "replay.cpp", "gemm_plan.cpp", "gemm_replay.cpp", "capi.cpp",
           "gemm_capi.cpp", "kernels.hip", "gemm_kernels.hip", "gemm_inst_bf16_256.hip", "gemm_inst_bf16_128.hip",
           "gemm_inst_f16_256.hip", "gemm_inst_f16_128.hip", "gemm_inst_bf16_split.hip", "gemm_inst_f16_split.hip",
           "gemm_inst_bf16_stream.hip", "gemm_inst_f16_stream.hip", "gemm_inst_bf16_split_any.hip", "gemm_inst_f16_split_any.hip",
           "gemm_inst_bf16_stream_any.hip", "gemm_inst_f16_stream_any.hip",
           "gemm_inst_bf16_gather.hip", "gemm_inst_f16_gather.hip", "gemm_inst_bf16_leaves.hip", "gemm_inst_f16_leaves.hip",
           "gemm_inst_bf16_wide.hip", "gemm_inst_f16_wide.hip",
           "mx_plan.cpp", "mx_gemm_plan.cpp", "mx_capi.cpp", "mx_kernels.hip", "mx_gemm_kernels.hip",
           "mx_gemm_inst_direct_codes.hip", "mx_gemm_inst_direct_bf16.hip", "mx_gemm_inst_direct_f16.hip", "mx_gemm_inst_stream_codes.hip", "mx_gemm_inst_ring_codes.hip", "mx_gemm_inst_wide_bf16_k.hip", "mx_gemm_inst_wide_bf16_rows.hip",
           "mx_gemm_inst_wide_f16_k.hip", "mx_gemm_inst_wide_f16_rows.hip",
           "mx_gemm_inst_stream_bf16_k.hip", "mx_gemm_inst_stream_bf16_rows.hip", "mx_gemm_inst_stream_f16_k.hip", "mx_gemm_inst_stream_f16_rows.hip",
           "rope_plan.cpp", "mx_cache_plan.cpp", "mx_attention_plan.cpp", "rope_cache_capi.cpp", "rope_kernels.hip", "mx_cache_kernels.hip", "mx_attention_kernels.hip",
           "mx_attention_inst_few_bf16.hip", "mx_attention_inst_few_f16.hip", "mx_attention_inst_tile_bf16.hip", "mx_attention_inst_tile_f16.hip"]
HEADERS = ["layout.hpp", "algebra.hpp", "semimodule.hpp", "plan.hpp", "kernel_params.hpp", "gemm_plan.hpp", "gemm_params.hpp", "plan_cache.hpp", "kernarg.hpp"]
# header -> the only sources that include it
_TILE = ["gemm_inst_bf16_256.hip", "gemm_inst_bf16_128.hip", "gemm_inst_f16_256.hip", "gemm_inst_f16_128.hip"]
_SPLIT = ["gemm_inst_%s_split%s.hip" % (t, a) for t in ("bf16", "f16") for a in ("", "_any")]
_STREAM = ["gemm_inst_%s_stream%s.hip" % (t, a) for t in ("bf16", "f16") for a in ("", "_any")]
_GATHER = ["gemm_inst_%s_%s.hip" % (t, g) for t in ("bf16", "f16") for g in ("gather", "leaves")]
_MX_DIRECT = ["mx_gemm_inst_direct_%s.hip" % t for t in ("codes", "bf16", "f16")]
_MX_STREAM = ["mx_gemm_inst_stream_%s.hip" % t for t in ("codes", "bf16_k", "bf16_rows", "f16_k", "f16_rows")]
_MX_RING = ["mx_gemm_inst_ring_codes.hip"]
_MX_WIDE = ["mx_gemm_inst_wide_%s_%s.hip" % (t, k) for t in ("bf16", "f16") for k in ("k", "rows")]
_WIDE = ["gemm_inst_%s_wide.hip" % t for t in ("bf16", "f16")]
_MX_GEMM = _MX_DIRECT + _MX_STREAM + _MX_RING + _MX_WIDE + ["mx_gemm_plan.cpp", "mx_gemm_kernels.hip", "mx_capi.cpp"]
_ATTENTION_FEW = ["mx_attention_inst_few_%s.hip" % t for t in ("bf16", "f16")]
_ATTENTION_TILE = ["mx_attention_inst_tile_%s.hip" % t for t in ("bf16", "f16")]
_ATTENTION_DEVICE = _ATTENTION_FEW + _ATTENTION_TILE + ["mx_attention_kernels.hip"]
_ATTENTION = _ATTENTION_DEVICE + ["mx_attention_plan.cpp", "rope_cache_capi.cpp"]
_ROPE = ["rope_plan.cpp", "rope_kernels.hip", "rope_cache_capi.cpp"]
_CACHE = _ATTENTION + ["mx_cache_plan.cpp", "mx_cache_kernels.hip"]
_MX = _MX_GEMM + ["mx_plan.cpp", "mx_kernels.hip"] + _CACHE + _ROPE
KERNEL_HEADERS = {"lds_limit.hpp": _TILE + _SPLIT + _STREAM + _GATHER + _WIDE + _MX_DIRECT + _MX_STREAM + _MX_RING + _MX_WIDE + _ATTENTION_TILE + _ATTENTION_FEW + ["kernels.hip", "capi.cpp"],
                  "rope_params.hpp": _ROPE, "rope_plan.hpp": _ROPE, "mx_cache_params.hpp": _CACHE, "mx_cache_plan.hpp": _CACHE,
                  "mx_attention_params.hpp": _ATTENTION, "mx_attention_plan.hpp": _ATTENTION, "mx_attention_device.hpp": _ATTENTION_DEVICE,
                  "mx_attention_few_kernel.hpp": _ATTENTION_FEW, "mx_attention_tile_kernel.hpp": _ATTENTION_TILE,
                  "mx_device.hpp": ["mx_kernels.hip", "mx_cache_kernels.hip", "rope_kernels.hip"],
                  "mx_params.hpp": _MX, "mx_plan.hpp": _MX, "mx_gemm_params.hpp": _MX_GEMM, "mx_gemm_plan.hpp": _MX_GEMM, "gemm_kernel.hpp": _TILE, "gemm_split_kernel.hpp": _SPLIT + _GATHER, "gemm_stream_kernel.hpp": _STREAM + _GATHER, "gemm_wide_kernel.hpp": _WIDE,
                  "gemm_device.hpp": _TILE + _SPLIT + _STREAM + _GATHER + _WIDE + _MX_DIRECT + _MX_STREAM + _MX_RING + _MX_WIDE + _ATTENTION_DEVICE + ["mx_kernels.hip", "mx_cache_kernels.hip", "rope_kernels.hip"],
                  "mx_gemm_device.hpp": _MX_DIRECT + _MX_STREAM + _MX_RING + _MX_WIDE + _ATTENTION_DEVICE, "mx_gemm_ring_kernel.hpp": _MX_RING, "mx_gemm_wide_kernel.hpp": _MX_WIDE, "mx_gemm_direct_kernel.hpp": _MX_DIRECT, "mx_gemm_stream_kernel.hpp": _MX_STREAM}


def _hipcc():
    return os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


# kernels.hip: the leading scalar kernel arguments (up to 14 dwords) are preloaded into scalar registers at wavefront
# start where the firmware supports it; the compiler keeps a prologue that loads them for firmware that does not
EXTRA_FLAGS = {"kernels.hip": ["-mllvm", "-amdgpu-kernarg-preload-count=14"]}


def compile_command(source):
    return [_hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-I" + INCLUDE,
            # packed-FP32 instruction selection is switched off for all device code
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"] + EXTRA_FLAGS.get(source, []) + [
            "-c", os.path.join(CSRC, source), "-o", os.path.join(OBJ_DIR, source + ".o")]


def link_command():
    return [_hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB_PATH] + [os.path.join(OBJ_DIR, s + ".o") for s in SOURCES]


def build(force=True):
    """Compile the library: one object per source (in parallel), then link.  With force=False objects and
    library that are newer than every source and header are kept."""
    os.makedirs(OBJ_DIR, exist_ok=True)
    common = [os.path.join(CSRC, h) for h in HEADERS] + [os.path.join(INCLUDE, "layoutcopy.h")]
    newest_common = max(os.path.getmtime(d) for d in common)
    todo = []
    for s in SOURCES:
        obj = os.path.join(OBJ_DIR, s + ".o")
        src_time = max(newest_common, os.path.getmtime(os.path.join(CSRC, s)))
        for header, sources in KERNEL_HEADERS.items():
            if s in sources:
                src_time = max(src_time, os.path.getmtime(os.path.join(CSRC, header)))
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < src_time:
            todo.append(s)
    if todo:
        with ThreadPoolExecutor(max_workers=min(8, len(todo))) as pool:
            list(pool.map(lambda s: subprocess.check_call(compile_command(s), cwd=CSRC), todo))
    if todo or not os.path.exists(LIB_PATH):
        subprocess.check_call(link_command(), cwd=CSRC)
    return LIB_PATH


if __name__ == "__main__":
    print(build())
