"""The pieces of rows that the grouped dense layers load: inside their arrays, at whole words, and the right elements of them, checked on the host (row_pieces.hip)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def test_pieces_are_whole_words_inside_their_arrays(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    exe = str(tmp_path / "row_pieces")
    subprocess.check_call([hipcc, "--offload-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Wno-unused-function",
                           "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I",
                           os.path.join(ROOT, "paper_2305_09887_amd", "csrc"), os.path.join(HERE, "row_pieces.hip"), "-o", exe])
    r = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0, f"ended with {r.returncode}: {r.stdout}"
    assert r.stdout == "4510 cases\n"
