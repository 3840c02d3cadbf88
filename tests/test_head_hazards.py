"""The hazards of test_strip_hazards.py and test_product_hazards.py in the kernels of the one-head losses: MFMAs in inline assembly,
for [H, V] heads and in the products also the LDS reads, and stages that grad_W of few tokens waits for by count."""
import re
import subprocess

import pytest

from paper_2603_01875_amd import kdloss as K
from tests.test_product_hazards import early_uses, late_waits
from tests.test_strip_hazards import LLVM, _code_objects, hazards, parse


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    K.lib()
    found = {}
    for obj in _code_objects(K._LIB_PATH, str(tmp_path_factory.mktemp("code"))):
        text = subprocess.run([f"{LLVM}/llvm-objdump", "-d", "--no-show-raw-insn", obj], check=True, capture_output=True,
                              text=True).stdout
        for m in re.finditer(r"^([0-9a-f]+) <(\S*head_\w+_kernel\S*)>:\n((?:\t.*\n)+)", text, re.M):
            found[m[2]] = parse(m[3].splitlines(), int(m[1], 16))
    return found


def _of(kernels, name):
    return {k: v for k, v in kernels.items() if re.search(r"\d" + name, k)}


def test_logit_kernels(kernels):
    logit = {**_of(kernels, "head_stats_kernel"), **_of(kernels, "head_grad_kernel")}
    assert len(logit) == 8 + 8                # order x smoothing x kept; order x smoothing x parts
    for name, code in logit.items():
        assert sum(c.op.startswith("v_mfma") for c in code) >= 4 * 64, name
        assert hazards(code) == [], name
        if "ILb1E" in name:                   # [H, V]
            assert early_uses(code) == [], name


def test_few_tokens(kernels):
    few = _of(kernels, "head_few_kernel")
    assert len(few) == 4                      # 64, 128 tokens x smoothing
    for name, code in few.items():
        assert sum(c.op.startswith("v_mfma") for c in code) >= 2 * 4 * 4 * 3, name
        assert hazards(code) == [], name


def test_products(kernels):
    products = _of(kernels, "head_gw_kernel")
    assert len(products) == 24                # tiles x order x type x add
    for name, code in products.items():
        assert hazards(code) == [] and early_uses(code) == [], name
    grad_h = _of(kernels, "head_gh_few_kernel")
    assert len(grad_h) == 4                   # 64, 128 tokens x order
    for name, code in grad_h.items():
        assert hazards(code) == [] and early_uses(code) == [], name
    few = _of(kernels, "head_gw_few_kernel")
    assert len(few) == 4                      # order x add
    for name, code in few.items():
        barriers, late = late_waits(code)
        assert early_uses(code) == [] and barriers and late == [], name
