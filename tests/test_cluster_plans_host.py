"""Plans whose CTAs form clusters and allocate tensor memory: what two of them can hold of one SM.  A CTA
of a cluster waits for its peers, and an allocation waits for free columns, so clusters on two
streams must never fit an SM together with more than its 512 columns between them.  The planners are plain
C++: they are compiled into a small library and asked directly."""
import ctypes
import itertools
import os
import shutil
import subprocess

import pytest

import paper_1501_06633_b200 as mx
from paper_1501_06633_b200 import workloads as wl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1501_06633_b200", "csrc")
SM_BYTES, CTA_BYTES, COLUMNS = 228 * 1024, 1024, 512     # an SM's shared memory, a CTA's own share, tensor memory columns

DRIVER = r"""
#include "%(csrc)s/gemm8.h"
#include "%(csrc)s/plan.h"
using namespace maxdnn;
extern "C" int set_opt(const char* name, int v) { return set_option(name, v); }
extern "C" void reset_opts() { reset_options(); }
extern "C" int gemm8(const maxdnn_gemm8_desc* d, int sms, int32_t* out) {
  if (check_gemm8(d) != MAXDNN_OK) return -1;
  Gemm8Plan p;
  const int st = plan_gemm8(*d, sms, &p);
  if (st != MAXDNN_OK) return st;
  const int32_t v[12] = {p.mx, p.pair, p.swap, p.tile_n, p.chunk, p.bulk_c, p.staged_c, p.split, p.k_blocks, p.stages, p.grid, p.smem_bytes};
  for (int i = 0; i < 12; ++i) out[i] = v[i];
  return 0;
}
extern "C" int wgrad(const maxdnn_conv_desc* d, int elem_bytes, int sms, int32_t* out) {
  static WgradGeom g;
  const int st = plan_wgrad(dims_from(*d), elem_bytes, sms, 0, &g, 1);
  if (st != MAXDNN_OK) return st;
  out[0] = g.pair; out[1] = g.smem_bytes;
  return 0;
}
"""
FIELDS = ("mx", "pair", "swap", "tile_n", "chunk", "bulk_c", "staged_c", "split", "k_blocks", "stages", "grid", "smem_bytes")


@pytest.fixture(scope="module")
def planners(tmp_path_factory):
    cxx = os.environ.get("CXX", "g++")
    if not shutil.which(cxx):
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("planners")
    src, lib = at / "driver.cpp", at / "planners.so"
    src.write_text(DRIVER % {"csrc": CSRC})
    subprocess.run([cxx, "-std=c++17", "-O1", "-fPIC", "-shared", "-o", str(lib), str(src), os.path.join(CSRC, "plan.cpp"),
                    os.path.join(CSRC, "gemm8_plan.cpp")], check=True)
    so = ctypes.CDLL(str(lib))
    yield so
    so.reset_opts()


def gemm8_plan(so, *args, **kw):
    out = (ctypes.c_int32 * 12)()
    st = so.gemm8(ctypes.byref(mx.Gemm8Desc.make(*args, **kw)), 148, out)
    return None if st else dict(zip(FIELDS, out))


def columns(p):
    """Tensor memory columns of a product's CTA: accumulators, and scales where the tensor core applies them."""
    nt = p["tile_n"]
    if not p["mx"]:
        return max(32, 2 * nt)
    need = (2 if nt <= 224 else 1) * nt + 4 * (4 + 4 * -(-nt // 128))
    return max(64, 1 << (need - 1).bit_length())


def every_cluster_plan(so):
    """(columns, shared memory) of the plans of cluster kernels over sizes, types, layouts and pinned shapes."""
    found = set()
    sizes = [(1, 128, 128), (1, 4096, 4096), (40, 300, 1000), (130, 257, 129), (700, 520, 640), (2048, 4096, 4096), (4096, 4096, 128)]
    shapes = [(None, None, None)] + [(-1, c, s) for c in (16, 32, 64, 128, 256) for s in (2, 4, 8)] + [(1, c, 1) for c in (128, 192, 224, 256)]
    for (m, n, k), (pair, cols, split), ct, scale, major in itertools.product(
            sizes, shapes, (mx.DTYPE_F32, mx.DTYPE_BF16), (mx.DTYPE_E8M0, mx.DTYPE_F32), (mx.MAJOR_K, mx.MAJOR_MN)):
        so.reset_opts()
        for name, v in ((b"GEMM8_PAIR", pair), (b"GEMM8_COLS", cols), (b"GEMM8_SPLIT", split)):
            if v is not None:
                so.set_opt(name, v)
        p = gemm8_plan(so, m, n, k, c_type=ct, a_scale_type=scale, b_scale_type=scale, a_major=major, b_major=major,
                       b_block=mx.BLOCK_TILE)
        if p and (p["pair"] or p["split"] > 1):
            found.add((columns(p), p["smem_bytes"]))
    so.reset_opts()
    out = (ctypes.c_int32 * 2)()
    convs = [w.dims for w in wl.WORKLOADS.values()] + [(64, 8, 8, 4, 256, 1, 1, 0, 1.0), (64, 8, 8, 8, 512, 3, 1, 1, 1.0)]
    for dims in convs:
        d = mx.ConvDesc.make(*dims)
        for bytes_ in (4, 2):
            if so.wgrad(ctypes.byref(d), bytes_, 148, out) == 0 and out[0]:
                found.add((COLUMNS, out[1]))
        for kind in (mx.KERNEL_TF32, mx.KERNEL_BF16):
            for kc in (0, 8, 16):
                mx.set_option("UMMA_PAIR", 1)
                mx.set_option("UMMA_KC", kc)
                try:
                    info, _ = mx.conv_plan_query(d, kind)
                except mx.MaxdnnError:
                    continue
                if info.pair:
                    found.add((COLUMNS, info.smem_bytes))
    return found


def test_no_two_clusters_fit_an_sm_with_more_than_its_tensor_memory(planners):
    found = sorted(every_cluster_plan(planners))
    assert {c for c, _ in found} >= {32, 64, 128, 256, 512}
    least = {c: min(s for k, s in found if k == c) for c, _ in found}
    for many in range(2, 18):
        for group in itertools.combinations_with_replacement(sorted(least), many):
            if sum(group) > COLUMNS:
                assert sum(least[c] + CTA_BYTES for c in group) > SM_BYTES, (group, least)
    assert max(s for _, s in found) <= 227 * 1024


def test_which_products_store_by_bulk_copies(planners):
    """Whole 16 bytes at both ends of every row, tiles of 32 columns or more, neither split nor exchanged roles."""
    so = planners
    for ct, bytes_ in ((mx.DTYPE_F32, 4), (mx.DTYPE_BF16, 2), (mx.DTYPE_F16, 2)):
        for n, ldc in ((328, 328), (328, 344), (330, 336), (331, 344), (328, 330)):
            for pair, cols in ((-1, 32), (-1, 64), (-1, 128), (1, 128), (1, 192), (1, 224), (1, 256)):
                so.reset_opts()
                for name, v in ((b"GEMM8_PAIR", pair), (b"GEMM8_COLS", cols), (b"GEMM8_SPLIT", 1), (b"GEMM8_SWAP", 0)):
                    so.set_opt(name, v)
                p = gemm8_plan(so, 150, n, 300, c_type=ct, ldc=ldc)
                whole = n * bytes_ % 16 == 0 and ldc * bytes_ % 16 == 0
                assert (p["tile_n"], p["pair"]) == (cols, int(pair > 0)) and bool(p["bulk_c"]) == whole and p["staged_c"]
    so.reset_opts()
