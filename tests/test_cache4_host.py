"""The 4-bit form's restatement against its definition, and the refusals of its
entry points that need no GPU."""

import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import cache4_oracle as O4


def test_four_significant_bits_rounded_up():
    t = np.array([0.0, 1.0, 15.0, 15.5, 17.0, 0.3, 2.0 ** -20, 1.0000001, 61440.0, 61441.0], np.float32)
    want = np.array([0.0, 1.0, 15.0, 16.0, 18.0, 0.3125, 2.0 ** -20, 1.125, 61440.0, 65536.0], np.float32)
    np.testing.assert_array_equal(O4.four_bits_up(t), want)
    rng = np.random.default_rng(0)
    x = np.exp(rng.uniform(-30, 30, 10000)).astype(np.float32)
    y = O4.four_bits_up(x)
    m, _ = np.frexp(y)
    assert (m * 16 == np.rint(m * 16)).all() and (y >= x).all() and (y <= x * 1.125).all()


def test_held_values_are_near_and_exact_in_bf16():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((50, 128)) * np.exp(rng.uniform(-3, 3, (50, 1)))).astype(np.float32)
    code, step = O4.quantise(x)
    assert code.min() >= 0 and code.max() <= 15
    held = O4.values(code, step)
    # half a step from the nearest whole number of steps (the largest value at 7.5 steps included)
    assert (np.abs(held - x) <= 0.5 * np.repeat(step, 32, -1) * (1 + 2.0 ** -20)).all()
    bits = held.astype(np.float32).view(np.uint32)
    assert not (bits & 0xFFFF).any()
    np.testing.assert_array_equal(O4.unpack(O4.pack(code)), code)
    assert (O4.pack(code)[:, 0] & 15 == code[:, 0]).all()


def test_rotation_keeps_lengths():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((3, 64))
    a = rng.uniform(0, 6, (3, 16))
    for pairs in (False, True):
        y = O4.rotate(x, np.cos(a), np.sin(a), pairs, np.float64)
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        np.testing.assert_array_equal(y[:, 32:], x[:, 32:])
        back = O4.rotate(y, np.cos(a), -np.sin(a), pairs, np.float64)
        np.testing.assert_allclose(back, x, atol=1e-12)


def test_refusals_without_a_context(lib):
    none = lib.VP_ERR_NOT_INITIALIZED
    assert lib.lib.vp_append(None, 1, 1, *([None] * 10)) == none
    assert lib.lib.vp_append4(None, 1, 1, *([None] * 12)) == none
    assert lib.lib.vp_reserve4(None, 1) == none
    assert lib.lib.vp_attend4(None, 1, 1, *([None] * 9)) == none


ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA_INC = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")


def _run(source, tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists(os.path.join(CUDA_INC, "cuda.h")):
        pytest.skip("needs g++ and the CUDA headers")
    exe = tmp_path / "invariants"
    src = tmp_path / "invariants.cpp"
    src.write_text(source)
    subprocess.run([cxx, "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2605_31457_gb300", "csrc"),
                    "-I", CUDA_INC, str(src), "-o", str(exe)], check=True, capture_output=True, text=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "0 violations" in r.stdout


def test_line_of_vp_attend4(tmp_path):
    """The cut of the work (line_invariants.cpp) with vp_attend4's row blocks, CTAs and fixed parts."""
    with open(os.path.join(ROOT, "tests", "line_invariants.cpp")) as f:
        s = f.read()
    for old, new in [("block = R > kTcTile ? 2 * kTcTile : R,", "block = R <= 8 ? 8 : R <= 16 ? 16 : R <= 24 ? 24 : 32,"),
                     ("Hkv = pick(1, 8), fixed = (dec ? 1 : 2) * kTileUnits;\n", "Hkv = pick(1, 8);\n"),
                     ("const int ctas = pick(0, 1) ? 152 : pick(1, 320);",
                      "const int ctas = 152 * pick(1, 3), fixed = B * nqt * Hkv <= ctas / 4 ? 2 : 6; (void)dec;")]:
        assert s.count(old) == 1, old
        s = s.replace(old, new)
    _run(s, tmp_path)


def test_workspace_of_vp_attend4(tmp_path):
    _run(r"""
#include <cstdio>
#include "vp_cache4.h"
int fails = 0;
void check(bool ok, const char* what, long a, long b) { if (!ok && ++fails < 20) std::printf("FAIL %s: %ld %ld\n", what, a, b); }
int main() {
  using namespace vp;
  for (int batch : {1, 3, 64, 1000}) for (int Hkv : {1, 8}) for (int G : {1, 4, 16}) for (int D : {64, 128})
  for (int max_seq : {1, 127, 129, 20480, 1 << 20}) for (int max_new : {1, 5, 64, 4096}) for (int page : {0, 1, 8, 256})
  for (int dtype : {0, 1}) {
    if (max_new > max_seq) continue;
    const Layout4 w = layout4(batch, Hkv * G, Hkv, D, max_seq, max_new, dtype, page > 0, page ? page : 16, 152);
    const NewLayout n = new_layout(batch, Hkv * G, Hkv, D, max_seq, max_new, 0, 152);
    if (!stages(dtype, page > 0, page, (long)max_new * G)) {
      check(w.seqs == 0 && w.total == n.total, "no staged rows", max_new, G);
      continue;
    }
    const size_t one = (size_t)Hkv * w.rows * D * 2;
    check(w.seqs >= 1 && w.seqs <= batch && (w.seqs == 1 || w.seqs * 2 * one <= kStageBytes), "sequences", w.seqs, batch);
    check(w.rows >= max_seq && w.rows % (page ? page : 128) == 0, "rows", w.rows, max_seq);
    check((long)w.pages * (page ? page : 128) == w.rows, "pages", w.pages, w.rows);
    check(w.o_k >= n.total && w.o_k % 128 == 0 && w.o_v % 128 == 0 && w.o_table % 4 == 0, "offsets", w.o_k, w.o_v);
    check(w.o_v - w.o_k >= w.seqs * one && w.o_table - w.o_v >= w.seqs * one, "room", w.seqs, one);
    check(!page || w.total - w.o_table >= (size_t)w.seqs * w.pages * 4, "table", w.seqs, w.pages);
  }
  // Records and tickets of the largest grids: CTAs per SM times two records of up to 32 rows.
  const NewLayout n = new_layout(1, 8, 8, 64, 100, 1, 0, 152);
  check(n.o_lse - n.o_tk >= 3u * 152 * 4, "tickets", 0, 0);
  check(n.o_o - n.o_st >= 2u * 2 * 152 * 32 * 8 && n.o_o - n.o_st >= 2u * 3 * 152 * 8 * 8, "sums", 0, 0);
  check(n.total - n.o_o >= (size_t)2 * 2 * 152 * 32 * 64 * 4, "outputs", 0, 0);
  std::printf("%d violations\n", fails);
  return fails != 0;
}
""", tmp_path)
