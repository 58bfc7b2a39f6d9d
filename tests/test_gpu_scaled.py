"""The block-scaled e4m3 quantiser (codes and scales, equal) and product (within the bound that
its types give) on the GPU against plain 64-bit forms (ops_ref.py)."""
import math

import numpy as np
import pytest
import torch

import ops_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


def host(t):
    return t.cpu().numpy()


def ref_quantize(x, block_rows):
    rows, cols = x.shape
    kb, rb = -(-cols // 128), -(-rows // block_rows)
    vals, exps = np.empty((rows, cols)), np.empty((rb, kb), np.int64)
    for i in range(rb):
        for c in range(kb):
            at = np.s_[i * block_rows:(i + 1) * block_rows, 128 * c:128 * c + 128]
            exps[i, c] = e = R.exponent(x[at])
            vals[at] = R.round8(x[at] / 2.0 ** int(e))
    return vals, exps.T if block_rows == 1 else exps


@pytest.mark.parametrize("dtype", [BF, FP, F32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 4096), (3, 144), (127, 256), (129, 1040), (260, 128)])
def test_quantize(rows, cols, block_rows, dtype):
    from paper_2509_04185_amd import scaled_quantize
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.randn((rows, cols + 16), generator=g) * torch.exp(2 * torch.randn((1, cols + 16), generator=g))
    x = x.to(dtype).to(DEV)[:, :cols]           # strided rows
    codes, scale = scaled_quantize(x, block_rows=block_rows)
    torch.cuda.synchronize()
    vals, exps = ref_quantize(R.f64(x), block_rows)
    assert np.array_equal(host(scale).astype(np.float64), 2.0 ** exps.astype(np.float64))
    assert np.array_equal(R.VALUES[host(codes)], vals)


def test_quantize_special_values():
    from paper_2509_04185_amd import scaled_quantize
    x = torch.randn((9, 256), generator=torch.Generator().manual_seed(1))
    x[0, :128] = 0
    x[1, 0], x[1, 1], x[1, 2] = math.inf, -math.inf, math.nan
    x[2] = math.nan
    x[3] = 3e38
    x[4] = 1e-40                # below the smallest scale: all zeros but not NaN
    x[5, :] = 448.0
    x[6, :] = 448.0001
    x[7] *= 2.0 ** -95
    for t in (x.to(DEV), x.to(BF).to(DEV)):
        codes, scale = scaled_quantize(t)
        torch.cuda.synchronize()
        vals, exps = ref_quantize(R.f64(t), 1)
        assert np.array_equal(host(scale).astype(np.float64), 2.0 ** exps.astype(np.float64))
        assert np.array_equal(R.VALUES[host(codes)], vals, equal_nan=True)


def make(m, n, k, seed, stride=0, signed=False):
    g = torch.Generator().manual_seed(seed)
    kb = -(-k // 128)

    def codes(r, c):
        return (torch.randn((r, c), generator=g) * 110).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    def scales(*shape):
        s = torch.exp(torch.randn(shape, generator=g)) * 0.01
        return s * (torch.randint(0, 2, shape, generator=g) * 2 - 1) if signed else s
    a = codes(m, k + stride).to(DEV)[:, :k]
    return a, scales(kb, m).to(DEV), codes(n, k).to(DEV), scales(-(-n // 128), kb).to(DEV)


def check_matmul(m, n, k, dtype, seed=0, stride=0, out=None, edit=None, signed=False):
    from paper_2509_04185_amd import scaled_matmul
    print(f"[gpu] scaled matmul {m} x {n} x {k} {dtype}", flush=True)
    a, sa, b, sb = make(m, n, k, seed + m + n + k, stride, signed)
    if edit:
        edit(a, sa, b, sb)
    got = scaled_matmul(a, sa, b, sb, out_dtype=dtype, out=out)
    torch.cuda.synchronize()
    want, bound = R.matmul(host(a), host(sa), host(b), host(sb), dtype)
    share = R.worst(R.f64(got), want, bound)
    print(f"    largest error {share:.3f} of its bound", flush=True)
    assert share <= 1.0
    return got


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 33, 48, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300])
def test_matmul_rows(m):
    check_matmul(m, 256, 512, BF)
    check_matmul(m, 130, 384, F32)


@pytest.mark.parametrize("n", [1, 2, 3, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 255, 257, 385, 1000])
def test_matmul_columns(n):
    check_matmul(5, n, 256, FP)
    check_matmul(70, n, 272, BF)
    check_matmul(300, n, 256, F32)


@pytest.mark.parametrize("k", [16, 32, 64, 80, 112, 128, 144, 240, 256, 272, 400, 1024, 1040, 4112])
def test_matmul_depth(k):
    check_matmul(7, 200, k, F32)
    check_matmul(40, 129, k, F32)
    check_matmul(150, 300, k, F32, signed=True)
    check_matmul(520, 260, k, BF)


@pytest.mark.parametrize("dtype", [BF, FP, F32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,n,k", [(16, 4096, 4096), (33, 1024, 14336), (512, 512, 1024), (200, 6144, 512)])
def test_matmul_sizes_and_types(m, n, k, dtype):
    check_matmul(m, n, k, dtype, stride=32)


@pytest.mark.parametrize("m,n,k,dtype", [(4096, 3600, 272, BF), (3500, 4100, 128, FP), (300, 28672, 656, BF),
                                         (257, 49285, 144, BF), (1100, 4096, 400, F32)], ids=lambda v: str(v))
def test_matmul_large(m, n, k, dtype):
    """Products of many tiles: rows and columns around the tiles' ends against the plain form."""
    from paper_2509_04185_amd import scaled_matmul
    print(f"[gpu] scaled matmul {m} x {n} x {k} {dtype}", flush=True)
    a, sa, b, sb = make(m, n, k, m, stride=16)
    got = R.f64(scaled_matmul(a, sa, b, sb, out_dtype=dtype))
    torch.cuda.synchronize()

    def some(size):
        near = np.concatenate([np.arange(e - 4, e + 4) for e in range(0, size + 257, 256)] + [np.arange(0, size, 37)])
        return np.unique(near[(near >= 0) & (near < size)])[:700]
    rows, cols = some(m), some(n)
    rows, cols = rows[::max(1, len(rows) // 150)], np.concatenate([cols[:300], some(n)[-100:]])
    want, bound = R.matmul(host(a)[rows], host(sa)[:, rows], host(b)[cols], host(sb), dtype, cols=cols)
    share = R.worst(got[np.ix_(rows, cols)], want, bound)
    print(f"    largest error {share:.3f} of its bound", flush=True)
    assert share <= 1.0 and np.isfinite(got).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("m", [18, 33, 47, 64])
def test_matmul_few_rows_many_columns(m, dtype):
    """Both sides of the widths and depths at which 17 to 64 rows change their kernel."""
    check_matmul(m, 4096, 272, dtype)
    check_matmul(m, 4099, 144, dtype)
    check_matmul(m, 16, 4096, dtype)
    check_matmul(m, 17, 4112, dtype)


@pytest.mark.parametrize("m,n,k,dtype", [(3300, 4099, 144, FP), (3500, 4100, 656, BF), (2529, 6454, 320, FP)],
                         ids=lambda v: str(v))
def test_matmul_large_odd_widths(m, n, k, dtype):
    """The rows of the output begin at every alignment of the type."""
    test_matmul_large(m, n, k, dtype)


def test_matmul_large_strided_output():
    """256-row tiles into rows of a wider, oddly aligned output: nothing beside them is written."""
    from paper_2509_04185_amd import scaled_matmul
    a, sa, b, sb = make(3300, 3301, 144, 7)
    plain = scaled_matmul(a, sa, b, sb)
    wide = torch.full((3300, 3309), 5.0, dtype=BF, device=DEV)
    scaled_matmul(a, sa, b, sb, out=wide[:, 3:3304])
    assert torch.equal(wide[:, 3:3304], plain)
    assert bool((wide[:, :3] == 5).all()) and bool((wide[:, 3304:] == 5).all())


@pytest.mark.parametrize("m", [9, 70, 300])
def test_matmul_strided_output(m):
    """Rows of a wider, oddly aligned output: nothing beside them is written."""
    wide = torch.full((m, 300), 5.0, dtype=BF, device=DEV)
    check_matmul(m, 200, 256, BF, out=wide[:, 3:203])
    assert bool((wide[:, :3] == 5).all()) and bool((wide[:, 203:] == 5).all())
    wide = torch.full((m, 304), 5.0, dtype=F32, device=DEV)
    check_matmul(m, 203, 256, F32, out=wide[:, 4:207])
    assert bool((wide[:, :4] == 5).all()) and bool((wide[:, 207:] == 5).all())


@pytest.mark.parametrize("m", [9, 70, 300])
def test_matmul_nan_stays_in_its_row_and_column(m):
    def edit(a, sa, b, sb):
        a[3, 17] = 0x7f
        b[101, 200] = 0xff
    got = check_matmul(m, 160, 256, F32, edit=edit)
    nan = torch.isnan(got).cpu().numpy()
    assert nan[3].all() and nan[:, 101].all() and nan.sum() == m + 160 - 1


def test_matmul_zero_and_infinite_scales():
    def edit(a, sa, b, sb):
        sa[0, 2] = 0.0
        sa[1, 4] = 1e38
        sb[0, 0] = 1e-38
    check_matmul(9, 160, 256, F32, edit=edit)


def test_matmul_no_rows():
    from paper_2509_04185_amd import scaled_matmul, scaled_quantize
    a, sa, b, sb = make(0, 64, 128, 1)
    assert scaled_matmul(a, sa, b, sb).shape == (0, 64)
    codes, scale = scaled_quantize(torch.empty((0, 128), device=DEV))
    assert codes.shape == (0, 128) and scale.shape == (1, 0)


def test_quantize_then_matmul_is_near_the_plain_product():
    """Both together as a projection uses them, against the product of the unrounded matrices: every
    operand is off by at most 2^-4 of itself, or of the format's smallest step at the block's scale."""
    from paper_2509_04185_amd import scaled_matmul, scaled_quantize
    g = torch.Generator().manual_seed(4)
    x = torch.randn((33, 512), generator=g).to(BF).to(DEV)
    w = (0.02 * torch.randn((300, 512), generator=g)).to(BF).to(DEV)
    y = scaled_matmul(*scaled_quantize(x), *scaled_quantize(w, block_rows=128), out_dtype=F32)
    torch.cuda.synchronize()
    X, W = R.f64(x), R.f64(w)
    h = 2.0 ** -4
    bound = (np.abs(X) @ np.abs(W).T) * (2 * h + h * h) + 1e-3
    assert (np.abs(R.f64(y) - X @ W.T) <= bound).all()
