"""Register and scratch use of the kernels around the experts' products, from the
compiler's resource report (no GPU needed): none may use scratch memory, and those
that memory bounds keep the waves that hide its latency."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_34162_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SOURCES = ("sdp_embed", "sdp_norm", "sdp_route", "sdp_order", "sdp_experts")


@pytest.fixture(scope="module")
def report(tmp_path_factory):
    if not os.path.exists(HIPCC) and not shutil.which("hipcc"):
        pytest.skip("hipcc not available")
    out = tmp_path_factory.mktemp("layer_res")

    def one(name):
        return subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature",
                               "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c",
                               os.path.join(CSRC, name + ".hip"), "-o", str(out / (name + ".o")),
                               "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True,
                              check=True).stderr
    kernels, name = {}, None
    with ThreadPoolExecutor(len(SOURCES)) as pool:
        text = "\n".join(pool.map(one, SOURCES))
    for line in text.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            name = m.group(1)
            kernels[name] = {}
        m = re.search(r"(ScratchSize \[bytes/lane\]|Occupancy \[waves/SIMD\]): (\d+)", line)
        if m and name:
            kernels[name][m.group(1).split()[0]] = int(m.group(2))
    assert len(kernels) > 20
    return kernels


def test_no_scratch(report):
    bad = {k: v["ScratchSize"] for k, v in report.items() if v["ScratchSize"]}
    assert not bad, bad


@pytest.mark.parametrize("kernel,waves", [("k_norm_rowsIttLi1ELb1E", 7), ("k_norm_back_rowsIttLb0E", 4), ("k_route_lanesI", 5),
                                          ("k_gatherI", 8), ("k_combineILi64EttL", 8), ("k_combine_backI", 7),
                                          ("k_embed_tableItLi4E", 4), ("k_embed_piecesIttL", 4)])
def test_occupancy(report, kernel, waves):
    found = {k: v["Occupancy"] for k, v in report.items() if kernel in k}
    assert found and min(found.values()) >= waves, found
