"""Products behind a long kernel, and of microscaled 4-bit matrices over many tiles and at the ends of the scales' range."""
import numpy as np
import pytest

import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B
    import gpu_harness as G
    from test_gpu_kv import ints
    from test_gpu_mx4 import CODE, DEV, T, check_product, dev, product_case


def product_of_nvfp4():
    M, N, K, fmt = 300, 512, 512, R.NVFP4
    xc, xs, wc, ws, x, w = product_case(M, N, K, fmt, seed=1)
    xc, xs, wc, ws = (dev(a) for a in (xc, xs, wc, ws))
    out = torch.full((M, N), 7.0, dtype=torch.float32, device=DEV)
    return out, lambda: B.sqap_mx4_linear(xc, xs, None, M, wc, ws, None, N, K, fmt, out, N, B.SQAP_FP32)


def product_of_int4(flag):
    """More tiles of the weights than SMs (or pairs of them), so that a CTA has a second one."""
    M, N, K = 40, 19200 if flag == B.SQAP_L_FORCE_TCGEN05_TS else 38400, 512
    g = np.random.default_rng(2)
    w = G.pack(g.integers(-7, 8, (N, K)), np.full(N, 0.01))
    q, sc = dev(g.integers(0, 256, (M, K // 2)).astype(np.uint8)), torch.full((M,), 0.02, device=DEV)
    out = torch.zeros((M, N), dtype=torch.int32, device=DEV)
    size = B.sqap_workspace_bytes(M, N, K, flag)
    work = torch.empty(size + 256, dtype=torch.uint8, device=DEV)
    at = (work.data_ptr() + 255) // 256 * 256
    return out, lambda: (B.sqap_w4a4_linear(q, sc, M, w, None, out, N, B.SQAP_I32, flag, at, size), work)


def test_products_behind_a_kernel_that_takes_longer_than_their_waits():
    """A product's CTAs may be on the device while the kernel in front still runs; their limits on waiting (some 2 s) do not count that.
    In front: attention of 149 heads on 148 SMs, so that all but one of them are free for the time of one head."""
    H, D, P, heads = 149, 256, 128, 149
    code = torch.zeros(1, H, P, D, dtype=torch.int8, device=DEV)
    scale = torch.ones(1, H, device=DEV)
    cache = B.KvCache(code, code, scale, scale, B.SQAP_KV_INT8)
    nq = 9
    q = torch.zeros(nq, heads * D, dtype=torch.float16, device=DEV)
    out_a = torch.empty_like(q)

    def attention(n):
        table = torch.zeros(1, -(-n // P), dtype=torch.int32, device=DEV)
        lens, cu = ints([n]), ints([0, nq])
        torch.cuda.synchronize()
        t = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        t[0].record()
        B.sqap_kv_attention(cache, table, table.shape[1], 1, lens, cu, nq, n, q, heads * D, heads, 0.1, 0, out_a, heads * D, None, 0, None, 0)
        return table, t

    attention(1 << 17)
    torch.cuda.synchronize()
    table, t = attention(1 << 20)
    t[1].record()
    torch.cuda.synchronize()
    n = int((1 << 20) * 5200 / t[0].elapsed_time(t[1]))       # two heads, 2.6 s each, one after the other
    assert n < 1 << 30
    for make in (product_of_nvfp4, lambda: product_of_int4(B.SQAP_L_FORCE_TCGEN05_TS), lambda: product_of_int4(B.SQAP_L_FORCE_TCGEN05_PAIR)):
        out, call = make()
        keep = call()
        torch.cuda.synchronize()
        want = out.clone()
        out.zero_()
        table, t = attention(n)
        keep = call(), keep
        t[1].record()
        torch.cuda.synchronize()
        assert t[0].elapsed_time(t[1]) > 4400
        assert B.sqap_device_status() == B.SQAP_OK
        assert want.any() and torch.equal(out, want)


# one to four tokens are multiplied on CUDA cores, five on tensor cores
@pytest.mark.parametrize("M", [1, 2, 4, 5])
@pytest.mark.parametrize("x_exp,w_exp", [(125, -100), (120, -60), (-100, 100), (-120, 20), (125, -127)])
def test_power_of_two_scales_at_the_ends_of_their_range(M, x_exp, w_exp):
    """A product of scales that fits fp32 is right wherever the scales themselves lie."""
    N, K, fmt = 40, 256, R.MXFP4
    g = np.random.default_rng(M)
    xc, wc = (g.integers(0, 256, (r, K // 2)).astype(np.uint8) for r in (M, N))
    xs, ws = ((127 + e + g.integers(0, 3, (r, K // 32)) - (e > 100)).clip(0, 254).astype(np.uint8) for e, r in ((x_exp, M), (w_exp, N)))
    x, w = R.mx4_values(xc, xs, fmt), R.mx4_values(wc, ws, fmt)
    out = torch.full((M, N), 7.0, dtype=torch.float32, device=DEV)
    B.sqap_mx4_linear(dev(xc), dev(R.tile(xs, 0xFF)), None, M, dev(wc), dev(R.tile(ws, 0xFF)), None, N, K, fmt, out, N, B.SQAP_FP32)
    torch.cuda.synchronize()
    check_product(out.double().cpu().numpy(), x, w, "fp32", K)


# 64, 128 and 192 tokens a tile; two to seven tiles for each pair of CTAs of a B200, of one to five stages, the last one short or whole
@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
@pytest.mark.parametrize("M,N,K", [(200, 12300, 544), (330, 12300, 288), (1100, 5000, 1056), (700, 5000, 1280), (1100, 19000, 96), (60, 40000, 512)])
def test_products_of_several_tiles_to_a_pair(M, N, K, fmt):
    xc, xs, wc, ws, x, w = product_case(M, N, K, fmt, seed=M + N + K)
    args = [dev(a) for a in (xc, xs)], [dev(a) for a in (wc, ws)]
    ldo = (N + 7) // 8 * 8 + 8
    for dtype in ("fp32", "bf16"):
        got = []
        for _ in range(2):
            out = torch.full((M + 1, ldo), 7.0, dtype=T[dtype], device=DEV)
            B.sqap_mx4_linear(*args[0], None, M, *args[1], None, N, K, fmt, out, ldo, CODE[dtype])
            torch.cuda.synchronize()
            assert B.sqap_device_status() == B.SQAP_OK
            got.append(out)
        assert torch.equal(got[0], got[1])
        o = got[0].double().cpu().numpy()
        assert (o[M] == 7).all() and (o[:, N:] == 7).all()
        check_product(o[:M, :N], x, w, dtype, K)


@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
@pytest.mark.parametrize("M,N,K", [(1, 12280, 4096), (1, 12288, 4096), (1, 12304, 4096), (2, 4096, 6144), (2, 4104, 6144)])
def test_one_and_two_tokens_on_either_side_of_the_rule(M, N, K, fmt):
    xc, xs, wc, ws, x, w = product_case(M, N, K, fmt, seed=M + N + K)
    out = torch.full((M + 1, N), 7.0, dtype=torch.float32, device=DEV)
    B.sqap_mx4_linear(dev(xc), dev(xs), None, M, dev(wc), dev(ws), None, N, K, fmt, out, N, B.SQAP_FP32)
    torch.cuda.synchronize()
    o = out.double().cpu().numpy()
    assert (o[M] == 7).all()
    check_product(o[:M], x, w, "fp32", K)


@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
@pytest.mark.parametrize("M,N,K", [(1, 1, 32), (4, 1, 32), (5, 1, 32), (64, 3, 16384), (300, 1, 64), (70001, 20, 64)])
def test_products_of_the_smallest_and_tallest_sizes(M, N, K, fmt):
    xc, xs, wc, ws, x, w = product_case(M, N, K, fmt, seed=M + N + K)
    out = torch.full((M + 1, 24), 7.0, dtype=torch.float32, device=DEV)
    B.sqap_mx4_linear(dev(xc), dev(xs), None, M, dev(wc), dev(ws), None, N, K, fmt, out, 24, B.SQAP_FP32)
    torch.cuda.synchronize()
    assert B.sqap_device_status() == B.SQAP_OK
    o = out.double().cpu().numpy()
    assert (o[M] == 7).all() and (o[:, N:] == 7).all()
    check_product(o[:M, :N], x, w, "fp32", K)


@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
def test_quantizer_and_inverse_of_more_rows_than_a_grid_is_high(fmt):
    M, K = 70001, 96
    x = torch.randn(M, K, device=DEV)
    codes = torch.empty(M, K // 2, dtype=torch.uint8, device=DEV)
    sc = torch.full((B.sqap_mx4_scale_bytes(M, K, fmt),), 0x7F, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(x)
    B.sqap_mx4_quantize(x, B.SQAP_FP32, M, K, K, None, fmt, None, codes, sc)
    B.sqap_mx4_dequantize(codes, sc, M, K, fmt, None, out, K, B.SQAP_FP32)
    torch.cuda.synchronize()
    v, scale = R.mx4_quantize(x.double().cpu().numpy(), fmt)
    assert np.array_equal(R.E2M1[R.nibbles(codes.cpu().numpy())], v)
    want = (v.reshape(M, -1, R.block(fmt)) * scale[..., None]).reshape(M, K)
    assert np.array_equal(out.double().cpu().numpy(), want)
