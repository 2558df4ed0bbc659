"""Rows that do not exist among the rows of a CTA of the window attention (csrc/window_keys.cuh), on the host."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_rows_that_do_not_exist(tmp_path):
    exe = str(tmp_path / "window_rows")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-Wno-unknown-pragmas", "-o", exe,
                           os.path.join(HERE, "window_rows_host.cpp")])
    subprocess.run([exe], check=True, timeout=120)


def test_the_kernel_uses_them():
    """attn.cu hands the functions of the header no positions of its own making for rows that do not exist, and lets them call for no second pass."""
    attn = open(os.path.join(os.path.dirname(HERE), "paper_2506_05096_b200", "csrc", "attn.cu")).read()
    assert "st.lo = tok >= 0 ? tok - p.left : kNoRowLo; st.hi = tok >= 0 ? tok + p.right : kNoRowHi;" in attn
    assert "__reduce_max_sync(0xffffffffu, st.lo), __reduce_min_sync(0xffffffffu, st.hi)" in attn
    assert "counts = st.lo != kNoRowLo;" in attn and "counts && !(tile_sum <= kTileSumLimit)" in attn
