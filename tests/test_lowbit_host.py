"""What the microscaled 4-bit and key/value cache calls refuse, and the sizes they report. No kernel is launched."""
import numpy as np
import pytest

import lowbit_reference as R
from paper_2509_09090_b200 import binding as B


def test_mx4_scale_and_workspace_bytes():
    for rows, K in [(1, 32), (128, 64), (129, 64), (300, 11008), (1, 96)]:
        for fmt in (0, 1):
            nb = K // R.block(fmt)
            assert B.sqap_mx4_scale_bytes(rows, K, fmt) == -(-rows // 128) * -(-nb // 4) * 512
            n = B.sqap_mx4_workspace_bytes(rows, 64, K, fmt)
            assert n >= rows * K // 2 + B.sqap_mx4_scale_bytes(rows, K, fmt) and n % 256 == 0
    assert B.sqap_mx4_scale_bytes(0, 64, 0) == B.sqap_mx4_scale_bytes(4, 0, 0) == B.sqap_mx4_scale_bytes(4, 64, 2) == 0


def test_reference_scale_tiles_are_inverse():
    b = np.random.default_rng(0).integers(0, 256, (300, 11)).astype(np.uint8)
    assert np.array_equal(R.untile(R.tile(b), 300, 11), b)


INV, ALIGN, NOMEM, OK = B.SQAP_ERR_INVALID, B.SQAP_ERR_ALIGN, B.SQAP_ERR_NOMEM, B.SQAP_OK


@pytest.mark.parametrize("change,want", [
    (dict(M=0), OK), (dict(M=-1), INV), (dict(x=None), INV), (dict(codes=None), INV), (dict(scales=None), INV), (dict(K=0), INV),
    (dict(K=48), ALIGN), (dict(ldx=32), INV), (dict(ldx=68), ALIGN), (dict(x=8), ALIGN), (dict(codes=24), ALIGN),
    (dict(scales=8), ALIGN), (dict(dt=2), INV), (dict(dt=4), INV), (dict(fmt=2), INV), (dict(fmt=-1), INV)])
def test_mx4_quantize_refusals(change, want):
    a = dict(x=16, dt=0, M=4, K=64, ldx=64, ri=None, fmt=0, g=None, codes=16, scales=16, stream=None)
    a.update(change)
    assert B.lib().sqap_mx4_quantize(*a.values()) == want


@pytest.mark.parametrize("change,want", [
    (dict(M=0), OK), (dict(M=-1), INV), (dict(codes=None), INV), (dict(out=None), INV), (dict(K=40), ALIGN), (dict(ldo=32), INV),
    (dict(ldo=68), ALIGN), (dict(out=4), ALIGN), (dict(dt=2), INV), (dict(fmt=7), INV)])
def test_mx4_dequantize_refusals(change, want):
    a = dict(codes=16, scales=16, M=4, K=64, fmt=0, g=None, out=16, ldo=64, dt=1, stream=None)
    a.update(change)
    assert B.lib().sqap_mx4_dequantize(*a.values()) == want


@pytest.mark.parametrize("change,want", [
    (dict(M=0), OK), (dict(M=-1), INV), (dict(N=0), INV), (dict(K=0), INV), (dict(K=80), ALIGN), (dict(xc=None), INV),
    (dict(xs=None), INV), (dict(wc=None), INV), (dict(ws=None), INV), (dict(out=None), INV), (dict(xc=8), ALIGN), (dict(ws=4), ALIGN),
    (dict(ldo=64), INV), (dict(ldo=132), ALIGN), (dict(dt=2), INV), (dict(fmt=3), INV)])
def test_mx4_linear_refusals(change, want):
    a = dict(xc=16, xs=16, gx=None, M=4, wc=16, ws=16, gw=None, N=128, K=64, fmt=0, out=16, ldo=128, dt=0, stream=None)
    a.update(change)
    assert B.lib().sqap_mx4_linear(*a.values()) == want


@pytest.mark.parametrize("change,want", [
    (dict(M=0), OK), (dict(M=-1), INV), (dict(x=None), INV), (dict(xdt=2), INV), (dict(ldx=8), INV), (dict(ldx=65), ALIGN),
    (dict(work=None), INV), (dict(work=8), ALIGN), (dict(bytes=100), NOMEM), (dict(wc=None), INV), (dict(K=33), ALIGN)])
def test_mx4_quantize_linear_refusals(change, want):
    a = dict(x=16, xdt=0, M=4, ldx=64, ri=None, gx=None, wc=16, ws=16, gw=None, N=128, K=64, fmt=0, out=16, ldo=128, dt=0, work=16,
             bytes=1 << 20, stream=None)
    a.update(change)
    assert B.lib().sqap_mx4_quantize_linear(*a.values()) == want
