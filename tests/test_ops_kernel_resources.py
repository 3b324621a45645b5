"""Register and scratch use of the training operators' kernels, from the
compiler's resource report (no GPU needed): none may use scratch memory, the
256 x 256 matrix tiles must leave two waves to a SIMD, and a row of logits held
in 1,024 threads' registers four."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_34162_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def report(tmp_path_factory):
    if not os.path.exists(HIPCC) and not shutil.which("hipcc"):
        pytest.skip("hipcc not available")
    out = tmp_path_factory.mktemp("ops_res")

    def one(name):
        return subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature",
                               "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c",
                               os.path.join(CSRC, name + ".hip"), "-o", str(out / (name + ".o")),
                               "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True,
                              check=True).stderr
    kernels, name = {}, None
    with ThreadPoolExecutor(3) as pool:
        text = "\n".join(pool.map(one, ("sdp_qk", "sdp_grouped", "sdp_distill")))
    for line in text.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            name = m.group(1)
            kernels[name] = {}
        m = re.search(r"(ScratchSize \[bytes/lane\]|Occupancy \[waves/SIMD\]): (\d+)", line)
        if m and name:
            kernels[name][m.group(1).split()[0]] = int(m.group(2))
    assert len(kernels) > 50
    return kernels


def test_no_scratch(report):
    bad = {k: v["ScratchSize"] for k, v in report.items() if v["ScratchSize"]}
    assert not bad, bad


def test_occupancy(report):
    for k, v in report.items():
        if "k_grouped_stream" in k or ("k_grouped" in k and "Li256E" in k):
            assert v["Occupancy"] >= 2, (k, v)
        if "k_distill_resident" in k and "Li1024E" in k:
            assert v["Occupancy"] >= 4, (k, v)
        if "k_qk_tokens" in k:
            assert v["Occupancy"] >= 3, (k, v)
