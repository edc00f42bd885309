"""What test_gated_assembly.py asks of the bfloat16 kernels, of the binary16 ones: the same source built on its own, with the same loads and products
written in assembly."""
import re
import subprocess

import pytest

from paper_2507_07149_amd import build
from tests.test_gated_assembly import (test_buffers_of_loads_come_from_the_scalar_unit, test_loops_of_products_wait_for_their_own_loads,  # noqa: F401
                                       test_sums_are_left_alone_next_to_their_products)


@pytest.fixture(scope="module")
def functions():
    """{kernel: its instructions, without comments; labels end in a colon}"""
    defines = next(s for s in build.SOURCES if s[1] == "gated_product_f16")[2]
    r = subprocess.run([build.HIPCC, *build.FLAGS, *defines, "--cuda-device-only", "-S", build.CSRC + "/gated_product.hip", "-o", "-"],
                       stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found = {}
    for body in re.split(r"\n\.Lfunc_end\d+:", r.stdout):
        if m := re.search(r"^(_Z\w*k_gated_\w+):.*$", body, re.M):
            lines = (line.split(";")[0].strip() for line in body[m.end():].splitlines())
            found[m.group(1)] = [s for s in lines if s and (not s.startswith(".") or s.endswith(":"))]
    products = [s for code in found.values() for s in code if s.startswith("v_mfma")]
    assert len(found) > 20 and products and all("_f16 " in s for s in products)
    return found
