"""Registers of the product kernels, as the compiler reports them (no GPU needed): a spill costs them more than any of their steps gains."""
import re
import shutil
import subprocess

import pytest

from paper_2601_22442_amd.build import HIPCC_FLAGS, PKG

FLAGS = [f for f in HIPCC_FLAGS if f not in ("-shared", "-Wall", "-Wextra")]
# name, vector registers that the resident waves leave: two waves a SIMD with 256, four with 128
LARGE = [(f"am::k_product_large<{a}, {b}>", 256) for a, b in (("false", "false"), ("false", "true"), ("true", "true"))]
SMALL = [(f"am::k_product<__bf16, 64, 64, 2, 2, {a}, {b}, true, {s}>", 128) for a, b in (("false", "false"), ("true", "true")) for s in (2, 4)]
MEDIUM = [("am::k_product<__bf16, 128, 128, 2, 2, false, true, true, 2>", 256), ("am::k_product_medium<true, true>", 256)]


@pytest.fixture(scope="module")
def reports(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    src = tmp_path_factory.mktemp("products") / "products.hip"
    src.write_text(f'#include "{PKG}/csrc/am_linear.h"\n' + "".join(f"template __global__ void {k}(const am::ProductArgs);\n" for k, _ in LARGE + SMALL + MEDIUM))
    out = subprocess.run(["hipcc", *FLAGS, "-c", "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-o", "/dev/null", str(src)],
                         capture_output=True, text=True, check=True).stderr
    found = [{k: int(v) for k, v in re.findall(r"remark: .*? (VGPRs|VGPRs Spill|ScratchSize)(?: \[\S+\])?: (\d+)", part)} for part in out.split("Function Name: ")[1:]]
    return dict(zip((k for k, _ in LARGE + SMALL + MEDIUM), found))


@pytest.mark.parametrize("kernel,limit", LARGE + SMALL + MEDIUM)
def test_products_stay_in_registers(reports, kernel, limit):
    r = reports[kernel]
    assert r["VGPRs"] <= limit and r["VGPRs Spill"] == 0 and r["ScratchSize"] == 0, r
