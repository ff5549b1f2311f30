"""relu's slope, value by value, where sums end near 0: 1 where A is greater than 0 in 64 bits, else 0.

The slopes are read off one by one: X has, behind the columns that A is formed of, a column of ones whose weights are 1 in Wu and 0 in Wg, so that U = 1, and a column of its own for
each row, 0 in both weights, so that dWg[f, that column] = dA[t, f] = dH U act' = act' for dH = 1.  0 and 1 have no rounding (fp16: dA is scaled by powers of two).
The products of 16-bit values are exact in 64 bits and their sums off by D 2^-53 of the terms' sizes: values of A that near 0 are not compared (there are none but exact zeros)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def pkg():
    import paper_2505_09326_amd as p
    p.load_library()
    return p


def _with_columns(data, wg, ones=1.0):
    """X, Wg, Wu around the data [T, n] and its weights [F, n]."""
    T, F = data.shape[0], wg.shape[0]
    X = torch.cat([data, torch.full((T, 1), ones, device=DEV, dtype=data.dtype), torch.eye(T, device=DEV, dtype=data.dtype)], 1).contiguous()
    Wg = torch.cat([wg, torch.zeros(F, T + 1, device=DEV, dtype=data.dtype)], 1).contiguous()
    Wu = torch.zeros_like(Wg)
    Wu[:, data.shape[1]] = 1.0 / ones
    return X, Wg, Wu


def _check(pkg, data, wg):
    """How many values a product in fp32 has on the other side."""
    T = data.shape[0]
    X, Wg, Wu = _with_columns(data, wg)
    dH = torch.ones(T, wg.shape[0], device=DEV, dtype=data.dtype)
    _, dWg, _ = pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "relu", want_dX=False, want_dWu=False)
    got = dWg[:, data.shape[1] + 1:].t().float()
    wt = wg.double().t().contiguous()
    A, size = data.double() @ wt, data.double().abs() @ wt.abs()
    sure = (A == 0) | (A.abs() > data.shape[1] * 2.0 ** -52 * size)
    assert (~sure).sum() == 0
    want = (A > 0).float()
    wrong = got != want
    assert not wrong.any(), f"{int(wrong.sum())} of {wrong.numel()} slopes, at A of {A[wrong][:5].tolist()} with terms of {size[wrong][:5].tolist()}"
    return int(((data.float() @ wg.float().t().contiguous() > 0) != (A > 0)).sum())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,n,F", [(3, 63, 200), (70, 257, 1000), (300, 1024, 2048), (500, 75, 4099)])
@pytest.mark.parametrize("offset", [0.0, 512.0])
def test_sums_that_cancel(pkg, T, n, F, dtype, offset):
    """An offset common to a row of X, which weights in pairs of opposite numbers take away again (as those of a layer behind a norm learn to)."""
    g = torch.Generator(device=DEV).manual_seed(T + n)
    t = TYPES[dtype]
    data = (offset + torch.randn(T, n, generator=g, device=DEV) * (8.0 if dtype == "bf16" and offset else 1.0)).to(t)
    half = torch.randn(F, n // 2, generator=g, device=DEV) * n ** -0.5
    wg = torch.cat([half, -half.flip(1)] + ([torch.zeros(F, 1, device=DEV)] if n % 2 else []), 1).to(t)
    if offset == 0:
        wg = torch.randn(F, n, generator=g, device=DEV).to(t)
    _check(pkg, data, wg)


def test_far_offset_in_fp32(pkg):
    """Beside terms of 10^4 the sums are of 1: a product in fp32 has hundreds of them on the other side."""
    g = torch.Generator(device=DEV).manual_seed(5)
    data = 10000.0 + torch.randn(400, 1024, generator=g, device=DEV)
    half = torch.randn(2500, 512, generator=g, device=DEV) / 32
    sides = _check(pkg, data, torch.cat([half, -half.flip(1)], 1))
    assert sides > 50


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T", [5, 150])
def test_sums_that_fp32_has_as_zero(pkg, T, dtype):
    """2^20 + 2^-20 - 2^20 and its like: 0 in fp32, and more or less than that or exactly that in 64 bits."""
    t = TYPES[dtype]
    data = torch.zeros(T, 80, device=DEV, dtype=t)
    data[:, 0], data[:, 1], data[:, 2], data[:, 40] = 1024.0, 2.0 ** -10, 1024.0, 2.0 ** -10
    data[T // 2] = 0                                           # (a row of zeros has slopes of 0)
    wg = torch.zeros(600, 80, device=DEV, dtype=t)
    wg[:, 0], wg[:, 2] = 1024.0, -1024.0
    wg[0::3, 1], wg[1::3, 1], wg[0::6, 40] = 2.0 ** -10, -(2.0 ** -10), -(2.0 ** -9)
    _check(pkg, data, wg)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sums_below_the_normal_numbers(pkg, dtype):
    """Values whose products fp32 has no bits left for."""
    g = torch.Generator(device=DEV).manual_seed(7)
    data, wg = (torch.randn(s, 40, generator=g, device=DEV).mul_(1e-23).to(TYPES[dtype]) for s in (90, 130))
    _check(pkg, data, wg)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_of_very_different_size(pkg, dtype):
    """Weights of one unit far above and of others far below the rest: each value goes by its own row's size."""
    g = torch.Generator(device=DEV).manual_seed(8)
    data, wg = torch.randn(200, 320, generator=g, device=DEV), torch.randn(700, 320, generator=g, device=DEV) / 16
    wg[::64] *= 2.0 ** -12 if dtype == "f16" else 2.0 ** -21
    wg[7] *= 2.0 ** 8 if dtype == "f16" else 2.0 ** 20
    wg[100:140] -= wg[100:140].mean(1, keepdim=True)
    data[50:60] += 64.0
    _check(pkg, data.to(TYPES[dtype]), wg.to(TYPES[dtype]))


def _time(pkg, X, Wg, Wu, dH):
    call = lambda: pkg.sphattn_gated_ffn_bwd(X, Wg, Wu, dH, "relu")
    call()
    best = []
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        best.append(a.elapsed_time(b))
    return sorted(best)[1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_data_takes_much_longer(pkg, dtype):
    """Units whose weights have decayed cost what others do; where every sum is near 0 the fp64 instruction bounds the time (one value at a time it was hundreds of times the
    products').  The bounds are several times what was measured: 1.0 and, for all sums near 0, 2.6 in bf16 and 1.9 in fp32."""
    g = torch.Generator(device=DEV).manual_seed(9)
    t = TYPES[dtype]
    T, D, F = 2048, 1024, 2048
    X, dH = torch.randn(T, D, generator=g, device=DEV).to(t), torch.randn(T, F, generator=g, device=DEV).to(t)
    Wg, Wu = (torch.randn(F, D, generator=g, device=DEV).mul_(1 / 32).to(t) for _ in range(2))
    usual = _time(pkg, X, Wg, Wu, dH)
    decayed = Wg.clone()
    decayed[::64] *= 2.0 ** -24
    assert _time(pkg, X, decayed, Wu, dH) < 2 * usual
    even = X.clone()
    even[:, 1::2] = even[:, 0::2]
    pairs = Wg.clone()
    pairs[:, 1::2] = -pairs[:, 0::2]                           # all sums are 0
    worst = _time(pkg, even, pairs, Wu, dH)
    print(f"{dtype}: usual {usual * 1e3:.0f} us, all sums 0 {worst * 1e3:.0f}")
    assert worst < 10 * usual
    # (in bf16 the sums in 64 bits are 0 whatever their order, of products of 16 bits; of fp32's 48 bits a sum's order decides what is left of 2^-53)
    _, dWg, _ = pkg.sphattn_gated_ffn_bwd(even, pairs, Wu, dH, "relu")
    assert dtype == "f32" or (dWg == 0).all()
