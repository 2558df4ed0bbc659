"""Which key tiles a CTA of the window attention walks over, and which keys of a tile a row sees (csrc/window_keys.cuh), on the host."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_window_keys(tmp_path):
    exe = str(tmp_path / "window_keys")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-Wno-unknown-pragmas", "-o", exe,
                           os.path.join(HERE, "window_keys_host.cpp")])
    subprocess.run([exe], check=True, timeout=120)
