"""Registers of the optimizer's and the layer norm's kernels, from the metadata of the library's own code objects: none spills
vector registers but the widest backward pass in float32, whose sixteen waves have 128 each, and AdamW's have at most 64, eight
waves per SIMD."""
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


def test_nothing_spills(kernels):
    of = {n: r for n, r in kernels.items() if re.search(r"k_(adamw|gradient_norm|layer_norm)", n)}
    assert len(of) > 200
    spills = {n: r[1] for n, r in of.items() if r[1]}
    assert all(re.search(r"k_layer_norm_backwardIffLi1024", n) and s <= 16 for n, s in spills.items()), spills


@pytest.mark.parametrize("pattern", ["k_adamwI", "k_adamw_codedI", "k_adamw_valuesI", "k_gradient_normI"])
def test_eight_waves_per_simd(kernels, pattern):
    of = {n: r for n, r in kernels.items() if pattern in n}
    assert of and not {n: r for n, r in of.items() if r[0] > 64 or r[1]}
