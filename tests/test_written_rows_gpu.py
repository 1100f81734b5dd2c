"""vp_append, vp_append4 and vp_attend4 refuse rows to write that overlap: caches and
outputs whose stride along an axis of more than one element is below a row."""

import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA_INC = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")


def test_rows_apart(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists(os.path.join(CUDA_INC, "cuda.h")):
        pytest.skip("needs g++ and the CUDA headers")
    src, exe = tmp_path / "apart.cpp", tmp_path / "apart"
    src.write_text("""
#include "vp_cache4.h"
int main() {
  using vp::rows_apart;
  bool ok = rows_apart(4096, 64, 128, 3, 2, 9, 64) && rows_apart(0, 0, 0, 1, 1, 1, 64) && rows_apart(0, 64, 128, 1, 2, 9, 64);
  ok = ok && !rows_apart(0, 64, 128, 2, 2, 9, 64) && !rows_apart(4096, 0, 128, 3, 2, 9, 64) && !rows_apart(4096, 64, 0, 3, 2, 9, 64);
  ok = ok && !rows_apart(4096, 56, 128, 3, 2, 9, 64) && !rows_apart(4096, 64, 8, 3, 2, 9, 64) && rows_apart(4096, 8, 128, 3, 1, 9, 64);
  return ok ? 0 : 1;
}
""")
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "paper_2605_31457_gb300", "csrc"), "-I", CUDA_INC,
                    str(src), "-o", str(exe)], check=True, capture_output=True, text=True)
    assert subprocess.run([str(exe)], timeout=60).returncode == 0


def _but(struct, **fields):
    copy = type(struct).from_buffer_copy(struct)
    for name, value in fields.items():
        setattr(copy, name, value)
    return copy


@pytest.mark.gpu
@pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
@pytest.mark.parametrize("page", [0, 16])
def test_appending(lib, four, page):
    from tests.test_append_gpu import Append
    vp = lib
    a = Append(vp, (8, 2), 64, "bf16", lens=(30, 12), n_new=2, four=four, page=page)
    call = vp.vp_append4 if four else vp.vp_append
    good = dict(batch=2, n_new=2, q=vp.rows(a.q_in), k=vp.rows(a.k_in), v=vp.rows(a.v_in), seq_len=a.seq,
                rotation=a.rotation, q_out=vp.rows(a.q_out), k_cache=a.kc, v_cache=a.vc)
    before = [y.clone() for c in a.caches for y in c]
    fields = ["code_stride_", "scale_stride_"] if four else ["stride_"]
    for name, cache in (("k_cache", a.kc), ("v_cache", a.vc)):
        for field in fields:
            for axis in "bht":
                for value in (0, 16 if field[0] == "c" else 8 if field[:2] == "st" else None):
                    if value is not None:
                        change = {name: _but(cache, **{field + axis: value})}
                        assert call(a.ctx, **{**good, **change}, check=False) == vp.VP_ERR_INVALID_ARG, (field, axis, value)
                        assert "stride" in vp.vp_last_error(a.ctx)
    assert call(a.ctx, **{**good, "q_out": _but(good["q_out"], stride_h=56)}, check=False) == vp.VP_ERR_INVALID_ARG
    torch.cuda.synchronize()
    for y, z in zip([y for c in a.caches for y in c], before):
        assert torch.equal(y, z)
    a.run()


@pytest.mark.gpu
@pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
def test_axes_of_one_element_may_have_any_stride(lib, four):
    from tests.test_append_gpu import Append
    a = Append(lib, (8, 1), 64, "bf16", lens=(30,), n_new=2, four=four)
    for cache in (a.kc, a.vc):
        if four:
            cache.code_stride_b = cache.code_stride_h = cache.scale_stride_b = cache.scale_stride_h = 0
        else:
            cache.stride_b = cache.stride_h = 0
    a.run()


@pytest.mark.gpu
def test_attention(lib):
    from tests.test_attend4_gpu import Case
    vp = lib
    a = Case(vp, (8, 2), 64, "bf16", lens=(64, 40), n_new=2)
    for change in (dict(stride_b=0), dict(stride_n=0), dict(stride_h=0), dict(stride_h=56), dict(stride_n=8)):
        assert vp.vp_attend4(a.ctx, 2, 2, vp.rows(a.q), a.kc, a.vc, a.seq, a.vis, _but(vp.rows(a.out), **change),
                             check=False) == vp.VP_ERR_INVALID_ARG
    assert torch.isnan(a.out).all()
    a.run()
