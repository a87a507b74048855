"""Registers of dropout's, the residual norm's and the loss's kernels, from the metadata of the library's own code objects: none spills vector
registers but the backward pass of teams of 512 in 16 bits (four) and, once per tile, the loss's largest tiles (ten, backward and forward with
smoothing), and nothing that a CU has to hold several of fills it alone."""
import os
import re
import shutil
import subprocess

import pytest

import paper_1908_06077_amd as nuq

LLVM = "/opt/rocm/llvm/bin"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
pytestmark = pytest.mark.skipif(not shutil.which("llvm-readelf", path=LLVM), reason="no LLVM tools")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("code")
    bundle, code = str(tmp / "bundle"), str(tmp / "code")
    subprocess.run([LLVM + "/llvm-objcopy", "--dump-section", ".hip_fatbin=" + bundle, nuq.library_path(), os.devnull], check=True)
    with open(bundle, "rb") as f:
        parts = f.read().split(MAGIC)[1:]                    # one per source file
    found = {}
    for part in parts:
        with open(bundle, "wb") as f:
            f.write(MAGIC + part)
        subprocess.run([LLVM + "/clang-offload-bundler", "--unbundle", "--type=o", "--input=" + bundle, "--output=" + code,
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
        notes = subprocess.run([LLVM + "/llvm-readelf", "--notes", code], check=True, capture_output=True, text=True).stdout
        for name, vgprs, spilled in re.findall(
                r"\.name: +(\S+)\n(?:(?! *\.name:).*\n)*? *\.vgpr_count: +(\d+)\n *\.vgpr_spill_count: +(\d+)", notes):
            found[name] = (int(vgprs), int(spilled))
    return found


@pytest.mark.parametrize("pattern, least", [("k_dropout", 10), ("k_residual_norm", 200), ("k_loss", 70)])
def test_nothing_spills(kernels, pattern, least):
    of = {n: r for n, r in kernels.items() if pattern in n}
    assert len(of) >= least
    most = {r"k_residual_norm_backwardIDF16.*Li512ELi8ELi8E": 4, r"k_loss_gradientI.*Li256ELi256E": 10, r"k_loss_logitsI.*Li256ELi256E.*ELb1E": 10}
    spills = {n: r[1] for n, r in of.items() if r[1] > max((m for p, m in most.items() if re.search(p, n)), default=0)}
    assert not spills


def test_waves_per_simd(kernels):
    """Eight for dropout; two for the products' largest tiles, whose workgroups of eight waves have a CU each."""
    dropout = {n: r for n, r in kernels.items() if "k_dropout" in n}
    assert not {n: r for n, r in dropout.items() if r[0] > 64}
    tiles = {n: r for n, r in kernels.items() if re.search(r"k_loss.*ProductTile.*Li256ELi256E", n)}
    assert len(tiles) >= 8 and not {n: r for n, r in tiles.items() if r[0] > 256}
