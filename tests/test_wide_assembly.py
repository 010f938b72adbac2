"""The products of wide layers, read from their assembly: their results never go to scratch memory, the compiler waits for no load of its own among the matrix
instructions (it would wait for the fetches of the next slabs with it), and the wait states around fetches in assembler are kept."""
import os
import re
import subprocess

import pytest

from paper_2305_09887_amd import build
from test_assembler_waits import too_near


@pytest.fixture(scope="module", params=["gated_dense", "dense_residual"])
def assembly(request, tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("wide") / "device.s"
    subprocess.check_call([build.HIPCC, *build.FLAGS, "-Wno-unused-function", "--offload-device-only", "-S", os.path.join(build.CSRC, request.param + ".hip"), "-o", str(out)])
    return out.read_text()


def kernels(text):
    """(name, lines) of the products."""
    for m in re.finditer(r"^(_ZN3tma\d+wide_(?:gemm|split)_kernel\w+):.*?s_endpgm", text, re.S | re.M):
        yield m.group(1), m.group(0).splitlines()


def blocks_of_products(lines):
    block, found = [], []
    for line in lines + [".LBB"]:
        if line.startswith(".LBB"):
            if sum("v_mfma" in x for x in block) >= 4:
                found.append(block)
            block = []
        block.append(line.split(";")[0].strip())
    return found


def waits(lines):
    return [x for block in blocks_of_products(lines) for x in block if x.startswith("s_waitcnt") and "vmcnt" in x and "lgkmcnt(0)" not in x]


def test_a_planted_wait_is_seen():
    product = ["v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]"] * 4
    assert len(waits([".LBB0_1:"] + product + ["s_waitcnt vmcnt(0)"] + product)) == 1
    assert not waits([".LBB0_1:"] + product + ["s_waitcnt lgkmcnt(3)"] + product)


def test_products(assembly):
    seen = 0
    for name, lines in kernels(assembly):
        seen += 1
        assert blocks_of_products(lines), name
        assert not waits(lines), name
        assert not any("scratch_" in x for x in lines), name
    assert seen >= 6


def test_distances(assembly):
    wrong, fetches, products = too_near(assembly)
    assert fetches > 50 and products > 50
    assert not wrong, wrong[:5]
