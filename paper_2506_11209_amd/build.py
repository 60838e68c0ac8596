"""Build libwsgemm.so (HIP, gfx950) in-tree.

    python -m paper_2506_11209_amd.build [--jobs N]

Generates one translation unit per group of kernel instantiations (so hipcc
runs in parallel), compiles them and the C-ABI host code with hipcc for
gfx950, and links ``paper_2506_11209_amd/libwsgemm.so``.  The per-kernel
register / LDS / spill report of the compiler goes to
``paper_2506_11209_amd/_build/resource_usage.txt``.
"""
from __future__ import annotations

import argparse
import concurrent.futures as cf
import os
import re
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libwsgemm.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# Every HIP file is compiled for gfx950 only.  Packed fp32 VALU ops are kept
# out of the generated code.
HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-x", "hip",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + CSRC, "-I" + os.path.join(ROOT, "include"), "-I" + BUILD,
]

# The 8-bit path and the routing of tokens to experts (ws_fp8.h, ws_experts.h).
OPERATOR_SOURCES = ["ws_fp8_product.hip", "ws_fp8_quantize.hip", "ws_experts.hip"]

# Kernel modes (KernelMode in ws_gemm_kernel.hpp): the GEMM and the
# calibration kernels of the performance model.
MODE_GEMM, CALIB_MODES = 0, (1, 2, 3, 4, 5)  # load A, load B, math, epilogue-only, load A+B


def instances():
    """(TM, TN, TK, consumer_waves, producer_waves, split, bf16, trace, mode,
    general) tuples that get a kernel.  Every configuration has a plain GEMM
    kernel and a general twin (shapes the tiles do not divide, the alpha /
    beta epilogue and 16-bit outputs); bf16 ones also get an event-traced twin
    (selected by ws_gemm_set_trace) and, for the arrangements the calibration
    covers, the calibration kernels of the performance model
    (ws_gemm_create_calibration)."""
    out = []
    # (consumer waves, producer waves, split): 1:1 and 2:1 with one or four
    # consumer waves; 2:1 at eight waves (two groups of two producer waves)
    arrangements = ((1, 1, 1), (4, 4, 1), (1, 2, 2), (4, 8, 2), (4, 4, 2))
    for bf16 in (1, 0):
        for nc, np_, split in arrangements:
            for tk in (32, 64):
                if nc == 1:
                    tiles = ((32, 32), (64, 64))
                else:
                    tiles = ((64, 64), (64, 128), (128, 64), (128, 128), (128, 256), (256, 128))
                for tm, tn in tiles:
                    out.append((tm, tn, tk, nc, np_, split, bf16, 0, MODE_GEMM, 0))
                    out.append((tm, tn, tk, nc, np_, split, bf16, 0, MODE_GEMM, 1))
                    if bf16:
                        out.append((tm, tn, tk, nc, np_, split, bf16, 1, MODE_GEMM, 0))
                        if nc == 4 and np_ == 4 * split:
                            out += [(tm, tn, tk, nc, np_, split, bf16, 0, m, 0) for m in CALIB_MODES]
    # Eight consumer waves (two per SIMD) and four producer waves, one group
    # (1:1) or two (2:1): 256 x 256 tiles of 128 x 64 wave tiles.
    for bf16 in (1, 0):
        for split in (1, 2):
            for tk in (32, 64):
                out.append((256, 256, tk, 8, 4, split, bf16, 0, MODE_GEMM, 0))
                out.append((256, 256, tk, 8, 4, split, bf16, 0, MODE_GEMM, 1))
                if bf16:
                    out.append((256, 256, tk, 8, 4, split, bf16, 1, MODE_GEMM, 0))
                    out += [(256, 256, tk, 8, 4, split, bf16, 0, m, 0) for m in CALIB_MODES]
    # Synchronous kernel (no producer waves): the same tiles, plus 256x256
    # whose 128x128 wave tiles fit once no producer shares the SIMD.
    for bf16 in (1, 0):
        for tk in (32, 64):
            tiles = [((tm, tn), 1) for tm, tn in ((32, 32), (64, 64))]
            tiles += [((tm, tn), 4) for tm, tn in ((64, 64), (64, 128), (128, 64), (128, 128),
                                                     (128, 256), (256, 128), (256, 256))]
            for (tm, tn), nc in tiles:
                out.append((tm, tn, tk, nc, 0, 0, bf16, 0, MODE_GEMM, 0))
    return out


def _generate(n_units: int) -> list[str]:
    os.makedirs(BUILD, exist_ok=True)
    inst = instances()
    units = [inst[i::n_units] for i in range(n_units)]
    paths = []
    for u, group in enumerate(units):
        lines = ["// generated by paper_2506_11209_amd/build.py -- do not edit",
                 '#include "ws_gemm_kernel.hpp"', '#include "ws_sync_kernel.hpp"',
                 '#include "ws_gemm_registry.hpp"',
                 "namespace wsg {",
                 "extern const KernelEntry kInstances%d[];" % u,
                 "extern const int kInstances%dCount;" % u,
                 "const KernelEntry kInstances%d[] = {" % u]
        lines += [("  WSG_ENTRY(%d, %d, %d, %d, %d, %d, %d, %d, %d, %d)," % t) if t[4] else
                  ("  WSG_SYNC_ENTRY(%d, %d, %d, %d, %d)," % (t[0], t[1], t[2], t[3], t[6]))
                  for t in group]
        lines += ["};", "const int kInstances%dCount = %d;" % (u, len(group)), "}  // namespace wsg", ""]
        p = os.path.join(BUILD, "ws_gemm_instances_%d.hip" % u)
        _write_if_changed(p, "\n".join(lines))
        paths.append(p)
    inc = ["// generated by paper_2506_11209_amd/build.py -- do not edit", "namespace wsg {"]
    for u in range(n_units):
        inc += ["extern const KernelEntry kInstances%d[];" % u, "extern const int kInstances%dCount;" % u]
    inc += ["}  // namespace wsg", "static const wsg::KernelTable kAllTables[] = {"]
    inc += ["  {wsg::kInstances%d, wsg::kInstances%dCount}," % (u, u) for u in range(n_units)]
    inc += ["};", "static const int kNumTables = %d;" % n_units, ""]
    _write_if_changed(os.path.join(BUILD, "ws_gemm_instances.inc"), "\n".join(inc))
    return paths


def _write_if_changed(path: str, text: str) -> None:
    if os.path.exists(path):
        with open(path) as f:
            if f.read() == text:
                return
    with open(path, "w") as f:
        f.write(text)


def _compile(src: str, obj: str, report: bool) -> tuple[str, str]:
    cmd = [HIPCC] + HIP_FLAGS + ["-c", src, "-o", obj]
    if report:
        cmd.insert(1, "-Rpass-analysis=kernel-resource-usage")
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, r.stderr[-6000:]))
    return src, r.stderr


def _parse_reports(reports: list[str]) -> list[dict]:
    rows = []
    cur = {}
    for text in reports:
        for line in text.splitlines():
            m = re.search(r"Function Name: (\S+)", line)
            if m:
                cur = {"name": m.group(1)}
                rows.append(cur)
                continue
            for key in ("VGPRs", "AGPRs", "ScratchSize", "Occupancy", "LDS Size", "SGPRs"):
                m = re.search(r"remark: .*\b%s(?: \[bytes/lane\])?: (\d+)" % re.escape(key), line)
                if m and cur:
                    cur[key] = int(m.group(1))
    return rows


_GEMM_NAME = re.compile(r"ws_gemm_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELb(\d)ELb(\d)ELi(\d+)ELb(\d)E")
_SYNC_NAME = re.compile(r"ws_sync_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELb(\d)E")


def _resource_table(rows: list[dict]) -> str:
    """C table of the registers every compiled kernel allocates, keyed like
    the kernel registry; the host planner derives occupancy from it."""
    entries = []
    for r in rows:
        name = r.get("name", "")
        m = _GEMM_NAME.search(name)
        if m:
            key = tuple(int(x) for x in m.groups())
        else:
            m = _SYNC_NAME.search(name)
            if not m:
                continue
            tm, tn, tk, nc, bf16 = (int(x) for x in m.groups())
            key = (tm, tn, tk, nc, 0, 0, bf16, 0, 0, 0)
        entries.append(key + (r.get("VGPRs", 0), r.get("AGPRs", 0)))
    entries.sort()
    lines = ["// generated by paper_2506_11209_amd/build.py -- do not edit",
             "static const wsg::KernelResources kResources[] = {"]
    lines += ["  {%d, %d, %d, %d, %d, %d, %d, %d, %d, %d, %d, %d}," % e for e in entries]
    lines += ["};", "static const int kNumResources = %d;" % len(entries), ""]
    return "\n".join(lines)


def _summarise(rows: list[dict]) -> str:
    out = []
    for r in rows:
        out.append("%-90s VGPR=%-4s AGPR=%-4s SGPR=%-4s scratch=%-5s occ=%s" % (
            r.get("name"), r.get("VGPRs"), r.get("AGPRs"), r.get("SGPRs"), r.get("ScratchSize"),
            r.get("Occupancy")))
    return "\n".join(out) + "\n"


def build(jobs: int | None = None, n_units: int = 32, verbose: bool = True) -> str:
    """Compile every HIP source for gfx950 and link libwsgemm.so; returns its path."""
    if not os.path.exists(HIPCC):
        raise RuntimeError("hipcc not found at %s" % HIPCC)
    units = _generate(n_units)
    jobs = jobs or min(16, os.cpu_count() or 4)
    api_src = os.path.join(CSRC, "ws_gemm_api.cpp")
    host_srcs = [api_src, os.path.join(CSRC, "ws_model.cpp")]
    host_jobs = [(h, os.path.join(BUILD, os.path.basename(h)[:-4] + ".o")) for h in host_srcs]
    kernel_jobs = [(u, u[:-4] + ".o") for u in units]
    kernel_jobs += [(os.path.join(CSRC, n), os.path.join(BUILD, n[:-4] + ".o")) for n in OPERATOR_SOURCES]
    reports = []
    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        # kernels first: the host API is compiled against their register table
        for f in [ex.submit(_compile, s, o, True) for s, o in kernel_jobs]:
            src, err = f.result()
            reports.append(err)
        rows = _parse_reports(reports)
        with open(os.path.join(BUILD, "resource_usage.txt"), "w") as f:
            f.write(_summarise(rows))
        _write_if_changed(os.path.join(BUILD, "ws_gemm_resources.inc"), _resource_table(rows))
        for f in [ex.submit(_compile, s, o, False) for s, o in host_jobs]:
            f.result()
    jobs_list = host_jobs + kernel_jobs
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + [o for _, o in jobs_list]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s" % r.stderr[-4000:])
    os.replace(tmp, LIB)
    if verbose:
        print("built %s (%d kernels)" % (LIB, len(instances())))
    return LIB


def clean() -> None:
    shutil.rmtree(BUILD, ignore_errors=True)
    if os.path.exists(LIB):
        os.remove(LIB)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--jobs", type=int, default=None)
    ap.add_argument("--clean", action="store_true")
    a = ap.parse_args()
    if a.clean:
        clean()
    build(a.jobs)
    sys.exit(0)
