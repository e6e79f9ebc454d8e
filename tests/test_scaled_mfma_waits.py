"""The waits after the scaled matrix instructions, over all paths of the kernels that use them, as
test_mfma_waits does for the others.  A 16x16x128 product of 4-bit operands takes four passes (16
cycles, the rate that a loop of them reaches), as a 16x16x32 one of bf16: eight wait states to the
first use of its result."""
import os

import pytest

from paper_2604_21026_amd import build
from tests import test_mfma_waits as waits

SHAPE = "16x16x128"


def plain(text):
    """A scaled product as an unscaled one of its shape: result and the first two operands first, as there."""
    return text.replace("v_mfma_scale_f32_%s_f8f6f4" % SHAPE, "v_mfma_f32_%s_f8f6f4" % SHAPE)


def test_a_missing_wait_is_found(monkeypatch):
    monkeypatch.setitem(waits.WAITS, SHAPE, 8)
    product = plain("v_mfma_scale_f32_16x16x128_f8f6f4 a[4:7], v[0:3], v[8:11], a[4:7], v12, v13 op_sel_hi:[0,0,0] cbsz:4 blgp:4")
    read = "v_accvgpr_read_b32 v20, a5"
    enough = [(0, product, None), (16, "s_nop 7", None), (20, read, None), (24, "s_endpgm", None)]
    assert waits.early_uses(enough) == []
    short = [(0, product, None), (16, "s_nop 6", None), (20, read, None), (24, "s_endpgm", None)]
    assert waits.early_uses(short) == [(20, "a5", 1)]


@pytest.mark.skipif(not os.path.exists(waits.OBJDUMP), reason="no llvm-objdump")
def test_no_kernel_uses_a_scaled_product_before_it_is_written(tmp_path, monkeypatch):
    monkeypatch.setitem(waits.WAITS, SHAPE, 8)
    if not os.path.exists(build.LIB):
        build.build()
    seen, bad = [], []
    for name, code in waits.kernels(build.LIB, str(tmp_path)):
        if not any("v_mfma_scale" in text for _, text, _ in code):
            continue
        assert all("cbsz:4 blgp:4" in text for _, text, _ in code if "v_mfma_scale" in text)
        seen.append(name)
        uses = waits.early_uses([(a, plain(text), target) for a, text, target in code])
        if uses:
            bad.append("%s: %d, first at %x: %s, %d states short" % ((name, len(uses)) + uses[0]))
    assert len(seen) >= 6 and all("gemm_mxfp4" in n for n in seen)
    assert not bad, "\n".join(bad)
