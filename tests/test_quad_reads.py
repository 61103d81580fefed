"""Which elements the 8-bit floating point quantizers read of rows that do not begin at a multiple of four: the kernels' own address
arithmetic (csrc/fp8.cuh), run on the host for every lane (no GPU)."""
import ctypes
import re
import subprocess

import pytest

from paper_1909_05840_b200 import build as qb_build

PROGRAM = r"""
#include "fp8.cuh"
#include <vector>

// How many elements outside x are read by the quads of the segments that are not read element by element; -1 where those leave out one of theirs.
static int outside(int64_t M, int64_t K, int shift, int width, int rows_per_warp) {
  const int64_t n = M * K;
  std::vector<char> seen(n);
  int bad = 0;
  for (int64_t m0 = 0; m0 < M; m0 += rows_per_warp)
    for (int64_t c = 0; c < K; c += width) {
      const int64_t rows = M - m0 < rows_per_warp ? M - m0 : rows_per_warp, first = m0 * K + c;
      const int left = (int)(K - c);
      if (qb::fp8_at_edge(first, first + (rows - 1) * K, left, width, n)) continue;
      for (int64_t base = first; base < first + rows * K; base += K) {
        const int off = (int)((base + shift) & 3);
        const auto quad = [&](int at) {
          for (int64_t k = base + at; k < base + at + 4; ++k) {
            if (k < 0 || k >= n) ++bad;
            else seen[k] = 1;
          }
        };
        seen.assign(n, 0);
        for (int j = 0; j < width / 128; ++j)
          for (int lane = 0; lane < 32; ++lane)
            if (qb::fp8_quad_at(j, lane, off) < left) quad(qb::fp8_quad_at(j, lane, off));
        if (qb::fp8_needs_behind(width, off, left)) quad(width - off);
        for (int k = 0; k < (left < width ? left : width); ++k)
          if (!seen[base + k]) return -1;
      }
    }
  return bad;
}
extern "C" int outside_rows(int64_t M, int64_t K, int shift) { return outside(M, K, shift, 512, 1); }
extern "C" int at_edge(int64_t base, int64_t K, int64_t n) { return qb::fp8_at_edge(base, base, (int)K, 512, n); }
extern "C" int outside_tile(int64_t M, int64_t K, int shift) { return outside(M, K, shift, 128, 16); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("quads")
    (d / "quads.cu").write_text(PROGRAM)
    subprocess.run([qb_build._nvcc(), "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC", "-shared",
                    "-I", str(qb_build.CSRC), str(d / "quads.cu"), "-o", str(d / "quads.so")], check=True)
    lib = ctypes.CDLL(str(d / "quads.so"))
    for f in (lib.outside_rows, lib.outside_tile):
        f.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int]
    lib.at_edge.argtypes = [ctypes.c_int64] * 3
    return lib


@pytest.mark.parametrize("M", [1, 2, 3, 5, 16, 17, 33])
def test_nothing_outside(lib, M):
    for K in [*range(1, 18), 125, 126, 127, 128, 129, 130, 131, 253, 384, 509, 510, 511, 512, 513, 514, 515, 1021, 1025]:
        for shift in range(4):
            assert lib.outside_rows(M, K, shift) == 0, (M, K, shift)
            assert lib.outside_tile(M, K, shift) == 0, (M, K, shift)


def test_few_are_read_one_by_one(lib):
    """Away from the ends of x nothing is: of 1,000 rows the first and the last."""
    for K in (384, 513):
        assert not any(lib.at_edge(r * K, K, 1000 * K) for r in range(1, 999)) and lib.at_edge(0, K, 1000 * K) and lib.at_edge(999 * K, K, 1000 * K)


def test_the_kernels_read_no_other_way():
    """Whole quads of rows that are all aligned, and those that the functions above name."""
    text = re.sub(r"//[^\n]*", "", (qb_build.CSRC / "quantize_fp8.cu").read_text())
    loads = [line.strip() for line in text.splitlines() if re.search(r"\bload\(", line)]
    assert loads == ["__device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }",
                     "if (left > j * 128) v[4 * s + j].load(p + j * 128);",
                     "if (at < left && left > 0) v[4 * s + j].load(p + at);",
                     "if (lane == 0 && fp8_needs_behind(512, off[s], left)) behind[s].load(p + 512 - off[s]);",
                     "for (int i = 0; i < 16; ++i) v[i].load(p + i * a.K);",
                     "if (i < rows && at < wide) v[i].load(r + at);",
                     "if (fp8_needs_behind(128, off, wide)) behind.load(r + 128 - off);"]
    assert text.count("fp8_at_edge(") == 2 and text.count("= fp8_quad_at(") == 2
