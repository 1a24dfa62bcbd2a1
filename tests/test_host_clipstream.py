"""The clipping kernels for large sets keep their loads past the caches, as
compiled for gfx950: where the compiler finds both forms of a load under one
run-time flag it merges them into the plain one, without a word."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("clip") / "clip.s")
    csrc = os.path.join(ROOT, "paper_2609_38767_amd", "csrc")
    subprocess.run([HIPCC, "-O3", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-x", "hip",
                    "--offload-device-only", "-S", os.path.join(csrc, "clip.hip"), "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()
    return {m[1]: m[2] for m in re.finditer(r"^(_Z\S*clip_\w+_kernelI\S*):(.*?)s_endpgm\s*\n\s*\.section", text,
                                            re.M | re.S)}


@pytest.mark.parametrize("name", ["clip_squares_kernel", "clip_scale_kernel"])
@pytest.mark.parametrize("stream", [True, False])
def test_loads(kernels, name, stream):
    body = [v for k, v in kernels.items() if f"{name}ILb{int(stream)}E" in k]
    assert len(body) == 1, sorted(kernels)
    loads = re.findall(r"global_load_dwordx4.*", body[0])
    past = [ln for ln in loads if re.search(r"\bnt\b", ln)]
    assert loads
    assert len(past) >= 16 if stream else not past  # eight in flight, two types at least
    assert not [ln for ln in re.findall(r"global_store_dwordx[24].*", body[0]) if re.search(r"\bnt\b", ln)]
