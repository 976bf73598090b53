"""Microscaled 4-bit quantizer, its inverse and the product against a plain 64-bit statement.

Tolerances. Codes and scales: equal (the reference makes the definition's fp32 roundings in the same places). Outputs of the
product: one rounding to the output type (half a step, finfo.eps / 2 relative) plus what the fp32 sums may lose:
the tensor core adds 64 products at a time and keeps at least 24 bits of the largest, so a sum of K products is off by at
most (K / 64 + 64) * 2^-23 * sum |x w|, and the split of K adds at most 8 more additions (2^-24 each). The multiplication
by the tensors' scales is two more roundings of 2^-24.
"""
import numpy as np
import pytest

import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B

DEV = "cuda:0"
T = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
CODE = {"fp16": 0, "bf16": 1, "fp32": 3}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def quantize(x, K, fmt, g=None, row_index=None, ldx=None):
    """x: torch tensor on the device, rows ldx apart. Returns (codes, raw scale bytes) as numpy, from buffers with a canary."""
    M = x.shape[0] if row_index is None else len(row_index)
    codes = torch.full((M + 1, K // 2), 0x5A, dtype=torch.uint8, device=DEV)
    n = B.sqap_mx4_scale_bytes(M, K, fmt)
    scales = torch.full((n + 64,), 0x7F, dtype=torch.uint8, device=DEV)
    dt = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 3}[x.dtype]
    gt = None if g is None else torch.tensor([g], dtype=torch.float32, device=DEV)
    ri = None if row_index is None else dev(np.asarray(row_index, np.int32))
    B.sqap_mx4_quantize(x, dt, M, K, ldx or x.stride(0), ri, fmt, gt, codes, scales)
    torch.cuda.synchronize()
    assert (codes[M] == 0x5A).all() and (scales[n:] == 0x7F).all()
    return codes[:M].cpu().numpy(), scales[:n].cpu().numpy()


def rows(M, K, dtype, seed=0, outliers=True):
    g = np.random.default_rng(seed)
    x = g.standard_normal((M, K))
    if outliers:
        x[:, g.integers(0, K, max(1, K // 50))] *= 30
    if M > 2:
        x[1] = 0                                   # a row of zeros
    if K >= 64:
        x[0, :64] = 0                              # blocks of zeros
    return torch.from_numpy(x).to(DEV).to(T[dtype])


@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("M,K", [(1, 32), (1, 64), (2, 96), (3, 160), (31, 224), (33, 4096), (128, 512), (129, 11008), (300, 32)])
def test_quantizer_codes_and_scales(M, K, dtype, fmt):
    x = rows(M, K, dtype, M + K)
    g = None if fmt == R.MXFP4 or M % 2 else 0.0071
    codes, raw = quantize(x, K, fmt, g)
    gv = 1.0 if g is None else float(np.float32(g))
    v, sc = R.mx4_quantize(x.double().cpu().numpy(), fmt, gv)
    nb = K // R.block(fmt)
    assert np.array_equal(R.scale_bytes_to_values(R.untile(raw, M, nb), fmt), sc)
    assert np.array_equal(R.E2M1[R.nibbles(codes)], v)
    pad = R.untile(raw, M, -(-nb // 4) * 4)[:, nb:]
    assert (pad == 0).all(), "bytes behind the last block of a row must be zero"


@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
def test_quantizer_ties_tiny_and_huge_values(fmt):
    """Every multiple of an eighth up to 7 (all halfway points among them) times scales from the smallest to the largest."""
    base = np.concatenate([np.arange(-56, 56) / 8.0, np.full(16, 6.0)])
    x = np.stack([base * s for s in (2.0 ** -14, 2.0 ** -8, 0.125, 1, 1.25, 3, 448, 2 ** 12, 2.0 ** -20)])
    xt = torch.from_numpy(x).to(DEV).float()
    codes, raw = quantize(xt, 128, fmt)
    v, sc = R.mx4_quantize(x, fmt)
    assert np.array_equal(R.scale_bytes_to_values(R.untile(raw, 9, 128 // R.block(fmt)), fmt), sc)
    assert np.array_equal(R.E2M1[R.nibbles(codes)], v)
    sub = torch.full((2, 64), 2.0 ** -133, dtype=torch.bfloat16, device=DEV)     # subnormal bf16
    codes, raw = quantize(sub, 64, fmt)
    v, sc = R.mx4_quantize(sub.double().cpu().numpy(), fmt)
    assert np.array_equal(R.E2M1[R.nibbles(codes)], v)


def test_quantizer_row_pitch_and_row_list():
    x = rows(40, 4096, "fp16", 3)
    part = x[:, 256:256 + 1024]
    codes, raw = quantize(part, 1024, R.NVFP4, ldx=4096)
    v, _ = R.mx4_quantize(part.double().cpu().numpy(), R.NVFP4)
    assert np.array_equal(R.E2M1[R.nibbles(codes)], v)
    idx = [39, 0, 0, 7, 21]
    codes, _ = quantize(part, 1024, R.NVFP4, row_index=idx, ldx=4096)
    assert np.array_equal(R.E2M1[R.nibbles(codes)], v[idx])


@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_dequantizer(dtype, fmt):
    M, K = 131, 352
    g = np.random.default_rng(5)
    codes = g.integers(0, 256, (M, K // 2)).astype(np.uint8)
    nb = K // R.block(fmt)
    byte = (g.integers(0, 0x60, (M, nb)) if fmt == R.NVFP4 else g.integers(115, 135, (M, nb))).astype(np.uint8)
    out = torch.full((M + 1, K + 8), 7.0, dtype=T[dtype], device=DEV)
    B.sqap_mx4_dequantize(dev(codes), dev(R.tile(byte, 0x7F)), M, K, fmt, torch.tensor([0.3], device=DEV), out, K + 8, CODE[dtype])
    torch.cuda.synchronize()
    ref = R.mx4_values(codes, byte, fmt, float(np.float32(0.3)))
    got = out.double().cpu().numpy()
    assert (got[M] == 7).all() and (got[:, K:] == 7).all()
    tiny = float(torch.finfo(T[dtype]).smallest_normal) * torch.finfo(T[dtype]).eps
    assert (np.abs(got[:M, :K] - ref) <= np.abs(ref) * (torch.finfo(T[dtype]).eps / 2 + 2.0 ** -23) + tiny / 2).all()


def product_case(M, N, K, fmt, seed=0, gx=None, gw=None):
    g = np.random.default_rng(seed)
    nb = K // R.block(fmt)
    xc, wc = (g.integers(0, 256, (r, K // 2)).astype(np.uint8) for r in (M, N))
    lo, hi = (0x18, 0x40) if fmt == R.NVFP4 else (122, 129)
    xs, ws = (g.integers(lo, hi, (r, nb)).astype(np.uint8) for r in (M, N))
    x, w = R.mx4_values(xc, xs, fmt, gx or 1.0), R.mx4_values(wc, ws, fmt, gw or 1.0)
    return xc, R.tile(xs, 0x7F if fmt == R.NVFP4 else 0xFF), wc, R.tile(ws, 0x7F if fmt == R.NVFP4 else 0xFF), x, w


def check_product(got, x, w, dtype, K):
    ref, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    fi = torch.finfo(T[dtype])
    tol = np.abs(ref) * (fi.eps / 2 + 2.0 ** -22) + mag * (K / 64 + 64 + 8) * 2.0 ** -23 + float(fi.smallest_normal) * fi.eps / 2
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} outputs off, first at {np.argwhere(bad)[0]}, worst {np.nanmax(np.abs(got - ref))}"


# sizes on either side of a tile, a stage (256), an MMA (64), a scale tile; K that ends in half an MMA
SHAPES = [(1, 128, 64), (1, 8, 32), (3, 130, 96), (16, 128, 256), (17, 257, 288), (16, 4096, 4096), (64, 384, 1024), (65, 128, 544),
          (127, 128, 11008), (129, 200, 512), (160, 512, 2048), (255, 129, 320), (256, 128, 256), (257, 130, 480), (288, 512, 4096),
          (600, 300, 1056), (1030, 520, 768), (1, 12288, 4096), (2, 1000, 16384)]


@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K, fmt):
    dtype = ("fp16", "bf16", "fp32")[(M + N + K // 32) % 3]
    gx, gw = (float(np.float32(0.02)), float(np.float32(0.5))) if fmt == R.NVFP4 else (None, None)
    xc, xs, wc, ws, x, w = product_case(M, N, K, fmt, M * 7 + N + K, gx, gw)
    if fmt == R.MXFP4 and dtype == "fp16" and K > 4096:
        dtype = "bf16"
    ldo = (N + 15) // 8 * 8
    out = torch.full((M + 1, ldo), 7.0, dtype=T[dtype], device=DEV)
    t = lambda v: None if v is None else torch.tensor([v], dtype=torch.float32, device=DEV)  # noqa: E731
    B.sqap_mx4_linear(dev(xc), dev(xs), t(gx), M, dev(wc), dev(ws), t(gw), N, K, fmt, out, ldo, CODE[dtype])
    torch.cuda.synchronize()
    assert B.sqap_device_status() == B.SQAP_OK
    got = out.double().cpu().numpy()
    assert (got[M] == 7).all() and (got[:, N:] == 7).all(), "wrote outside the output"
    check_product(got[:M, :N], x, w, dtype, K)


@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
@pytest.mark.parametrize("M,N,K", [(1, 512, 4096), (37, 300, 1056), (160, 256, 11008), (700, 384, 512)])
def test_fused_call_equals_the_two_calls(M, N, K, fmt):
    x = rows(M, K, "fp16", 11)
    _, _, wc, ws, _, _ = product_case(1, N, K, fmt, 4)
    wc, ws = dev(wc), dev(ws)
    gx, gw = torch.tensor([0.05], device=DEV), torch.tensor([0.25], device=DEV)
    codes = torch.empty(M, K // 2, dtype=torch.uint8, device=DEV)
    sc = torch.full((B.sqap_mx4_scale_bytes(M, K, fmt),), 0x7F, dtype=torch.uint8, device=DEV)
    a, b = (torch.full((M, N // 8 * 8 + 8), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.sqap_mx4_quantize(x, 0, M, K, K, None, fmt, gx, codes, sc)
    B.sqap_mx4_linear(codes, sc, gx, M, wc, ws, gw, N, K, fmt, a, a.stride(0), 1)
    n = B.sqap_mx4_workspace_bytes(M, N, K, fmt)
    work = torch.full((n,), 0x7F, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        B.sqap_mx4_quantize_linear(x, 0, M, K, None, gx, wc, ws, gw, N, K, fmt, b, b.stride(0), 1, work, n)
    torch.cuda.synchronize()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert B.sqap_device_status() == B.SQAP_OK


def test_weights_quantized_in_the_same_stream_right_before():
    """The weights are the output of the call in front: they may not be fetched before it is done."""
    M, N, K = 4, 4096, 4096
    fmt = R.NVFP4
    x, w = rows(M, K, "fp16", 1), [rows(N, K, "fp16", s) for s in (2, 3)]
    wc = torch.empty(N, K // 2, dtype=torch.uint8, device=DEV)
    ws = torch.empty(B.sqap_mx4_scale_bytes(N, K, fmt), dtype=torch.uint8, device=DEV)
    n = B.sqap_mx4_workspace_bytes(M, N, K, fmt)
    work = torch.empty(n, dtype=torch.uint8, device=DEV)
    got = []
    for fused in (True, False):
        for i in (0, 1, 0, 1):
            out = torch.empty(M, N, dtype=torch.float16, device=DEV)
            if not fused:
                B.sqap_mx4_quantize(x, 0, M, K, K, None, fmt, None, work, work.data_ptr() + M * K // 2)
            B.sqap_mx4_quantize(w[i], 0, N, K, K, None, fmt, None, wc, ws)
            if fused:
                B.sqap_mx4_quantize_linear(x, 0, M, K, None, None, wc, ws, None, N, K, fmt, out, N, 0, work, n)
            else:
                B.sqap_mx4_linear(work, work.data_ptr() + M * K // 2, None, M, wc, ws, None, N, K, fmt, out, N, 0)
            got.append(out)
    torch.cuda.synchronize()
    for i in range(8):
        assert torch.equal(got[i], got[i % 2])
    xv, _ = R.mx4_quantize(x.double().cpu().numpy(), fmt)
    assert not torch.equal(got[0], got[1])


def test_fused_call_in_a_graph_and_on_two_streams():
    M, N, K, fmt = 33, 640, 2048, R.MXFP4
    _, _, wc, ws, _, _ = product_case(1, N, K, fmt, 4)
    wc, ws = dev(wc), dev(ws)
    xs = [rows(M, K, "bf16", s) for s in (1, 2)]
    n = B.sqap_mx4_workspace_bytes(M, N, K, fmt)
    works = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [torch.empty(M, N, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ref = []

    def call(i, stream=None):
        B.sqap_mx4_quantize_linear(xs[i], 1, M, K, None, None, wc, ws, None, N, K, fmt, outs[i], N, 1, works[i], n, stream)

    for i in (0, 1):
        call(i)
        torch.cuda.synchronize()
        ref.append(outs[i].clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, s in enumerate(streams):
            call(i, s)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[i], ref[i]) for i in (0, 1))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(0)
        call(1)
    for o in outs:
        o.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(outs[i], ref[i]) for i in (0, 1))
    assert B.sqap_device_status() == B.SQAP_OK
