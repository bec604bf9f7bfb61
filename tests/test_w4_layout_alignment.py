"""gmlp_w4_quantize, _pack and _dequantize refuse bf16 arrays at odd addresses before any device work (a kernel that met one would fault)."""
import ctypes

import pytest
import torch

from paper_2606_26344_b200 import build as B
from paper_2606_26344_b200 import gmlp


@pytest.fixture(scope="module")
def lib():
    B.build_libgmlp()
    return gmlp.lib()


def status(entry, W, scales=None, zeros=None):
    m = gmlp.GmlpW4Matrix(0x10000, 0x20000, 0x30000 if zeros else None, 256, 64, 128, 0)
    return entry(ctypes.byref(gmlp.GmlpW4LayoutArgs(ctypes.sizeof(gmlp.GmlpW4LayoutArgs), 0, W, scales, zeros, m, None)))


def test_odd_addresses_are_refused(lib):
    assert status(lib.gmlp_w4_quantize, 0x1001) == gmlp.ERR_ALIGN
    assert status(lib.gmlp_w4_dequantize, 0x1001) == gmlp.ERR_ALIGN
    assert status(lib.gmlp_w4_pack, 0x1000, 0x2001) == gmlp.ERR_ALIGN


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where no kernel can be launched on them")
def test_elements_own_alignment_is_enough(lib):
    assert status(lib.gmlp_w4_quantize, 0x1002) == gmlp.ERR_ARCH
    assert status(lib.gmlp_w4_dequantize, 0x1002) == gmlp.ERR_ARCH
    assert status(lib.gmlp_w4_pack, 0x1001, 0x2002, 0x3001) == gmlp.ERR_ARCH
