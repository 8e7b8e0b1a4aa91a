"""Builds the C-ABI shared library in-tree with nvcc for sm_100a (no JIT cache, no torch headers)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "librap_b200.so")
LIB_DBG = os.path.join(HERE, "librap_b200_dbg.so")      # the same sources with -DRAP_DEBUG_BOUNDS (index checks in the kernels)
OBJ = os.path.join(HERE, "_build")
SOURCES = ["rap_api.cu", "rap_proj.cu", "rap_proj_tc.cu", "rap_attn.cu", "rap_attn_fast.cu", "rap_attn_scan.cu",
           "rap_lowrank.cu", "rap_lowrank_tc.cu", "rap_prefill.cu", "rap_prefill_tc.cu", "rap_q8.cu", "rap_q4.cu", "rap_window.cu",
           "rap_window_scan.cu", "rap_window_scan_long.cu", "rap_window_tc.cu"]
SCAN_PARTS = 8      # translation units the scan kernel's instantiations are spread over


def scan_shapes():
    """(G, P, d_v') head shapes the FP32-pipe scan is instantiated for (the tier behind the tensor-core scan,
    kept for cross-checks and for the low-rank comparator): the retain ratios of the D = 128 workloads (P, d_v'
    rounded independently) at G = 1..5 and full-width K with a pruned V for the comparator.  Shapes whose q
    registers alone would exceed 64 per thread are left to the run-time-shape kernel."""
    base = [(58, 115), (51, 102), (45, 90), (32, 64), (64, 128)]
    shapes = []
    for G in (1, 2, 3, 4, 5):
        shapes += [(G, P, dv) for P, dv in base]
    shapes += [(4, 64, dv) for dv in (115, 102, 90, 64)]

    def q_regs(G, P):
        kv = 1 if P % 2 else 2 if P % 4 else 4
        units = P // kv
        clu = (units + 7) // 8
        return G * clu * kv * 2

    out = []
    for sh in shapes:
        if sh not in out and q_regs(sh[0], sh[1]) <= 64:
            out.append(sh)
    return out


MMA_PARTS = 8


def mma_shapes():
    """(G, P, d_v') head shapes of the tensor-core (mma.sync) scan: the retain ratios of the D = 128 workloads
    (the unpruned cache included) at every group size up to 8, and every budget with d_v' = 2P for P = 16..64
    at G = 3, 4, 5 (what layer-adaptive allocation produces).  P = 32 and 64 with d_v' = 64, 128 are staged
    through swizzling tensor maps; the other multiples of 8 keep some bank conflicts in the fragment loads and
    are still faster here than on the FP32 pipes."""
    base = [(58, 115), (51, 102), (45, 90), (32, 64), (64, 128)]
    shapes = []
    for G in (1, 2, 3, 4, 5, 6, 7, 8):
        shapes += [(G, P, dv) for P, dv in base]
    for G in (3, 4, 5):
        shapes += [(G, P, 2 * P) for P in range(16, 65)]
    shapes.append((4, 64, 64))
    out = []
    for sh in shapes:
        if sh not in out:
            out.append(sh)
    return out


def mma_dyn_shapes():
    """Head shapes whose tensor-core scan is also built in the form that hands the last tiles of a long launch out at
    run time: the retain ratios of the D = 128 workloads at the group sizes of the shaped models."""
    base = [(58, 115), (51, 102), (45, 90), (32, 64), (64, 128)]
    return [(G, P, dv) for G in (3, 4, 5) for P, dv in base]


Q8_PARTS = 4


def q8_shapes():
    """(G, P, d_v') head shapes of the tensor-core scan over a quantised cache: the retain ratios of the D = 128
    workloads at the group sizes of the shaped models, and the 8B head shape at the other group sizes."""
    base = [(58, 115), (51, 102), (45, 90), (32, 64), (64, 128)]
    shapes = []
    for G in (3, 4, 5):
        shapes += [(G, P, dv) for P, dv in base]
    shapes += [(G, 45, 90) for G in (1, 2, 8)]
    return shapes


Q4_PARTS = 16


def q4_shapes():
    """(words per K row, words per V row, heads per lane) of the tensor-core scan over a 4-bit cache: every odd number of
    words up to 17 on both sides, so it covers every head of up to 128 dims and every group size up to 8."""
    words = range(3, 18, 2)
    return [(k, v, c) for c in (1, 2) for k in words for v in words]


def write_scan_sources():
    """Generated translation units: SCAN_PARTS files of instantiations and the lookup over them."""
    os.makedirs(OBJ, exist_ok=True)
    shapes = scan_shapes()
    names = []
    for k in range(SCAN_PARTS):
        mine = shapes[k::SCAN_PARTS]
        body = ['// generated by build.py: instantiations of the shape-specialised scan, part %d' % k,
                '#include "rap_attn_scan_kernel.cuh"', "namespace {",
                "template <int G, int WK, int DV> rap_scan_entry entry() {",
                "  return rap_scan_entry{G, WK, DV, ScanCfg<G, WK, DV>::SMEM, ScanCfg<G, WK, DV>::ST, STHREADS, 0,",
                "                        (const void*)attn_scan_kernel<G, WK, DV>, nullptr};", "}", "}  // namespace",
                "const rap_scan_entry* rap_scan_table_%d(int* n) {" % k,
                "  static const rap_scan_entry table[] = {"]
        body += ["    entry<%d, %d, %d>()," % sh for sh in mine]
        body += ["  };", "  *n = (int)(sizeof(table) / sizeof(table[0]));", "  return table;", "}", ""]
        names.append(_write_if_changed(os.path.join(OBJ, "scan_inst_%d.cu" % k), "\n".join(body)))
    mshapes = mma_shapes()
    for k in range(MMA_PARTS):
        mine = mshapes[k::MMA_PARTS]
        body = ['// generated by build.py: instantiations of the mma.sync scan, part %d' % k,
                '#include "rap_attn_mma_kernel.cuh"', "namespace {",
                "template <int G, int WK, int DV, bool WITH_DYN> rap_scan_entry entry() {",
                "  using C = MmaCfg<G, WK, DV>;",
                "  const void* dyn = nullptr;",
                "  if constexpr (WITH_DYN) dyn = (const void*)attn_mma_kernel<G, WK, DV, true>;",
                "  return rap_scan_entry{G, WK, DV, C::SMEM, C::ST, C::THREADS, C::TMA ? 1 : 0,",
                "                        (const void*)attn_mma_kernel<G, WK, DV, false>, dyn};",
                "}", "}  // namespace",
                "const rap_scan_entry* rap_mma_table_%d(int* n) {" % k,
                "  static const rap_scan_entry table[] = {"]
        dyn = mma_dyn_shapes()
        body += ["    entry<%d, %d, %d, %s>()," % (sh + ("true" if sh in dyn else "false",)) for sh in mine]
        body += ["  };", "  *n = (int)(sizeof(table) / sizeof(table[0]));", "  return table;", "}", ""]
        names.append(_write_if_changed(os.path.join(OBJ, "mma_inst_%d.cu" % k), "\n".join(body)))
    qshapes = q8_shapes()
    for k in range(Q8_PARTS):
        mine = qshapes[k::Q8_PARTS]
        body = ['// generated by build.py: instantiations of the tensor-core scan over a quantised cache, part %d' % k,
                '#include "rap_attn_q8_kernel.cuh"', "namespace {",
                "template <int G, int WK, int DV> rap_scan_entry entry() {",
                "  using C = Q8Cfg<G, WK, DV>;",
                "  return rap_scan_entry{G, WK, DV, C::SMEM, C::ST, C::THREADS, 0, (const void*)attn_q8_kernel<G, WK, DV>, nullptr};",
                "}", "}  // namespace",
                "const rap_scan_entry* rap_q8_table_%d(int* n) {" % k,
                "  static const rap_scan_entry table[] = {"]
        body += ["    entry<%d, %d, %d>()," % sh for sh in mine]
        body += ["  };", "  *n = (int)(sizeof(table) / sizeof(table[0]));", "  return table;", "}", ""]
        names.append(_write_if_changed(os.path.join(OBJ, "q8_inst_%d.cu" % k), "\n".join(body)))
    for k in range(Q4_PARTS):
        mine = q4_shapes()[k::Q4_PARTS]
        body = ['// generated by build.py: instantiations of the tensor-core scan over a 4-bit cache, part %d' % k,
                '#include "rap_attn_q4_kernel.cuh"', "namespace {",
                "template <int K, int V, int C> rap_q4_entry entry() {",
                "  return rap_q4_entry{K, V, C, Q4Cfg<K, V, C>::SMEM, Q4Cfg<K, V, C>::NW * 32, (const void*)attn_q4_kernel<K, V, C>};", "}", "}  // namespace",
                "const rap_q4_entry* rap_q4_table_%d(int* n) {" % k, "  static const rap_q4_entry table[] = {"]
        body += ["    entry<%d, %d, %d>()," % sh for sh in mine]
        body += ["  };", "  *n = (int)(sizeof(table) / sizeof(table[0]));", "  return table;", "}", ""]
        names.append(_write_if_changed(os.path.join(OBJ, "q4_inst_%d.cu" % k), "\n".join(body)))
    look = ['// generated by build.py: lookup over the instantiation tables', '#include "rap_internal.h"']
    look += ["const rap_q4_entry* rap_q4_table_%d(int* n);" % k for k in range(Q4_PARTS)]
    look += ["const rap_q4_entry* rap_q4_find(int k_words, int v_words, int heads_per_lane) {",
             "  typedef const rap_q4_entry* (*table_fn)(int*);",
             "  static const table_fn parts[] = {" + ", ".join("rap_q4_table_%d" % k for k in range(Q4_PARTS)) + "};",
             "  for (table_fn f : parts) {", "    int n = 0;", "    const rap_q4_entry* t = f(&n);",
             "    for (int i = 0; i < n; ++i)",
             "      if (t[i].k_words == k_words && t[i].v_words == v_words && t[i].heads_per_lane == heads_per_lane) return &t[i];",
             "  }", "  return nullptr;", "}"]
    look += ["const rap_scan_entry* rap_q8_table_%d(int* n);" % k for k in range(Q8_PARTS)]
    look += ["const rap_scan_entry* rap_q8_find(int G, int WK, int DV) {",
             "  typedef const rap_scan_entry* (*table_fn)(int*);",
             "  static const table_fn parts[] = {" + ", ".join("rap_q8_table_%d" % k for k in range(Q8_PARTS)) + "};",
             "  for (table_fn f : parts) {", "    int n = 0;", "    const rap_scan_entry* t = f(&n);",
             "    for (int i = 0; i < n; ++i)", "      if (t[i].G == G && t[i].WK == WK && t[i].DV == DV) return &t[i];",
             "  }", "  return nullptr;", "}"]
    look += ["const rap_scan_entry* rap_mma_table_%d(int* n);" % k for k in range(MMA_PARTS)]
    look += ["const rap_scan_entry* rap_mma_find(int G, int WK, int DV) {",
             "  typedef const rap_scan_entry* (*table_fn)(int*);",
             "  static const table_fn parts[] = {" + ", ".join("rap_mma_table_%d" % k for k in range(MMA_PARTS)) + "};",
             "  for (table_fn f : parts) {", "    int n = 0;", "    const rap_scan_entry* t = f(&n);",
             "    for (int i = 0; i < n; ++i)", "      if (t[i].G == G && t[i].WK == WK && t[i].DV == DV) return &t[i];",
             "  }", "  return nullptr;", "}"]
    look += ["const rap_scan_entry* rap_scan_table_%d(int* n);" % k for k in range(SCAN_PARTS)]
    look += ["const rap_scan_entry* rap_scan_find(int G, int WK, int DV) {",
             "  typedef const rap_scan_entry* (*table_fn)(int*);",
             "  static const table_fn parts[] = {" + ", ".join("rap_scan_table_%d" % k for k in range(SCAN_PARTS)) + "};",
             "  for (table_fn f : parts) {", "    int n = 0;", "    const rap_scan_entry* t = f(&n);",
             "    for (int i = 0; i < n; ++i)", "      if (t[i].G == G && t[i].WK == WK && t[i].DV == DV) return &t[i];",
             "  }", "  return nullptr;", "}", ""]
    names.append(_write_if_changed(os.path.join(OBJ, "scan_tables.cu"), "\n".join(look)))
    return names


def _write_if_changed(path, text):
    if not os.path.exists(path) or open(path).read() != text:
        with open(path, "w") as f:
            f.write(text)
    return path


def _stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "rap.h"), os.path.join(INCLUDE, "rap_debug.h"), os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def _stale_dbg():
    if not os.path.exists(LIB_DBG):
        return True
    t = os.path.getmtime(LIB_DBG)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "rap.h"), os.path.join(INCLUDE, "rap_debug.h"), os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build_debug(force=False):
    """The bounds-checking library librap_b200_dbg.so: every source compiled with -DRAP_DEBUG_BOUNDS, so that the index
    checks in the hand-indexed kernels are live (a failed check is recorded in the device status word as RAP_EBOUNDS
    and the access is skipped).  Same entry points; meant for tests."""
    if not force and not _stale_dbg():
        return LIB_DBG
    return build(force=True, debug=True)


def build(force=False, verbose=False, debug=False):
    """Compile every CUDA source into librap_b200.so (debug: into librap_b200_dbg.so with the index checks on);
    returns the library path."""
    global OBJ
    if not debug and not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a",
             "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    obj_release = OBJ
    if debug:
        flags += ["-DRAP_DEBUG_BOUNDS"]
        OBJ = OBJ + "_dbg"
    try:
        return _build_into(nvcc, flags, force, verbose, LIB_DBG if debug else LIB)
    finally:
        OBJ = obj_release


def _build_into(nvcc, flags, force, verbose, lib):
    os.makedirs(OBJ, exist_ok=True)

    generated = write_scan_sources()

    def compile_one(src):
        path = src if os.path.isabs(src) else os.path.join(CSRC, src)
        obj = os.path.join(OBJ, os.path.basename(src).replace(".cu", ".o"))
        headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
        deps = [path, os.path.join(INCLUDE, "rap.h"), os.path.join(INCLUDE, "rap_debug.h")] + headers
        if not force and os.path.exists(obj) and all(os.path.getmtime(d) <= os.path.getmtime(obj) for d in deps):
            return obj, None
        return obj, subprocess.run([nvcc] + flags + ["-c", path, "-o", obj], capture_output=True, text=True)

    with ThreadPoolExecutor(max_workers=os.cpu_count() or 8) as pool:     # one nvcc process per translation unit
        results = list(pool.map(compile_one, generated + SOURCES))
    for obj, res in results:
        if res is not None and (verbose or res.returncode):
            sys.stderr.write(res.stdout + res.stderr)
        if res is not None and res.returncode:
            raise RuntimeError("nvcc failed compiling " + obj)
    res = subprocess.run([nvcc, "-shared", "-o", lib] + [o for o, _ in results], capture_output=True, text=True)
    if res.returncode:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed linking " + os.path.basename(lib))
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    if "--debug" in sys.argv:
        print(build_debug(force="--force" in sys.argv))
