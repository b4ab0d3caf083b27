"""The operators between a layer's attention calls -- norm of the residual stream, rows in 8 bits, their products -- against plain forms in 64 bits (numpy).

Tolerances, from the arithmetic:
 * codes of the norm and of rows without activation, the stream's sum, and products: the operators fix every rounding, so bits are equal to those of the oracle
   with the same roundings.
 * scales: the norm's factor is formed in 64 bits and the scale rounded once, 2^-24 (the oracle's sum may be in another order, 64 bits again: 2^-40);
   that of other rows is one division, equal bits.
 * bf16 results of the norm: the factor, its product with h and that with the weight are rounded to fp32, 2^-24 each, and the result to bf16, 2^-8.
 * silu in fp32, x t / (1 + t) below zero and x / (1 + t) above, t = e^-|x|: the exponential 2^-22 (two units in the last place), its argument is exact, the product, the sum,
   the division and the product with the factor 2^-24 each: 2^-22 + 4 * 2^-24 = 2^-21 of the value.  A code is then within half a step, plus 127 times 2^-21 twice (of the value and of the
   row's largest) and the rounding of factor and product (2^-24 each): 0.5 + 1.4e-4 steps.
"""
import ctypes

import numpy as np
import pytest

from paper_2508_15919_amd import binding as hb
from paper_2508_15919_amd.synth import bf16_bits_to_f64, f32_to_bf16_bits

HALF_BF16 = 2.0 ** -8


def bf16(x):
    """Values rounded to bf16, in 64 bits."""
    return bf16_bits_to_f64(f32_to_bf16_bits(np.asarray(x, np.float32)))


def to_codes(v):
    """Rows of fp32 numbers -> codes and largest magnitudes, with the operators' roundings."""
    v = np.asarray(v, np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.maximum(np.abs(v).max(1, keepdims=True), np.float32(2.0 ** -100))
        bad = ~np.isfinite(v).all(1, keepdims=True)
        t = np.where(bad, np.float32(0), np.where(bad, np.float32(0), v) * (np.float32(127) / np.where(bad, np.float32(1), top)))
    return np.rint(t).astype(np.int8), np.where(bad, np.nan, top.astype(np.float64))


def device(torch, x, dtype=None):
    """bf16 values (64 bits on the host) on the GPU."""
    t = torch.from_numpy(np.ascontiguousarray(x))
    return t.to(dtype or torch.bfloat16).cuda()


def strided(torch, x, extra):
    """The rows of a tensor in a wider buffer, which holds NaN (or 77) beside them."""
    rows, cols = x.shape
    fill = 77 if x.dtype == torch.int8 else float("nan")
    wide = torch.full((rows, cols + extra), fill, dtype=x.dtype, device="cuda")
    wide[:, :cols] = x
    return wide


# ------------------------------------------------------------------ norm
def norm_oracle(x, residual, weight, eps):
    """Sum, result in 64 bits, codes, scales in 64 bits."""
    h = x if residual is None else bf16(x.astype(np.float32) + residual.astype(np.float32))
    with np.errstate(invalid="ignore", over="ignore"):
        r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + float(np.float32(eps)))
        codes, top = to_codes(h.astype(np.float32) * weight.astype(np.float32))
        return h, h * r * weight, codes, (top * r / 127.0)[:, 0]


def run_norm(torch, x, residual, weight, eps, extra=0, behind=2):
    rows, cols = x.shape
    dx = strided(torch, device(torch, x), extra)
    dr = None if residual is None else strided(torch, device(torch, residual), extra)
    total = None if residual is None else torch.full((rows + behind, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full((rows + behind, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    codes = torch.full((rows + behind, cols), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((rows + behind,), 7.0, dtype=torch.float32, device="cuda")
    norm = hb.make_norm(device(torch, weight), eps)
    hb.hfx_rms_norm(norm, rows, dx, cols + extra, dr, cols + extra, total, out, codes, scales, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for t, was in ((total, 7.0), (out, 7.0), (codes, 99), (scales, 7.0)):      # rows behind the last
        assert t is None or bool((t[rows:] == was).all())
    return [None if t is None else t[:rows].cpu().double().numpy() for t in (total, out, codes, scales)]


def check_norm(got, want):
    total, out, codes, scales = got
    h, y, want_codes, want_scales = want
    assert total is None or np.array_equal(total, h, equal_nan=True)
    assert np.array_equal(codes, want_codes)
    assert np.array_equal(np.isnan(scales), np.isnan(want_scales))
    fine = ~np.isnan(scales)
    assert (np.abs(scales - want_scales)[fine] <= (2.0 ** -24 + 2.0 ** -40) * want_scales[fine] + 2.0 ** -149).all()
    off = np.abs(out - y)[fine]
    assert (off <= (HALF_BF16 + 3 * 2.0 ** -24) * np.abs(y[fine]) + 2.0 ** -133).all()
    return fine


@pytest.mark.gpu
@pytest.mark.parametrize("with_residual", [True, False])
@pytest.mark.parametrize("rows,cols,extra", [(1, 16, 0), (3, 48, 8), (70, 512, 0), (5, 1024, 24), (4, 1040, 0), (33, 2048, 8), (2, 4096, 0), (3, 8192, 0), (2, 8208, 8),
                                             (1, 32768, 0), (2, 40016, 16), (1, 131056, 0), (1300, 4112, 8), (300, 16400, 0)])
def test_norm(rows, cols, extra, with_residual):
    import torch
    g = np.random.default_rng(rows * 131 + cols)
    x = bf16(g.standard_normal((rows, cols)))
    residual = bf16(3.0 * g.standard_normal((rows, cols))) if with_residual else None
    weight = bf16(1.0 + 0.3 * g.standard_normal(cols))
    fine = check_norm(run_norm(torch, x, residual, weight, 1e-6, extra), norm_oracle(x, residual, weight, 1e-6))
    assert fine.all()


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [64, 4096, 9008])
def test_norm_of_extreme_rows(cols):
    """Zeros, subnormal and largest numbers, squares past the range of 32 bits, one value among zeros, ties, and rows that are not finite beside all of them."""
    import torch
    g = np.random.default_rng(cols)
    x = bf16(g.standard_normal((12, cols)))
    weight = np.ones(cols)
    x[0] = 0.0
    x[1] = 0.0
    x[1, 5] = -2.0 ** -133                                      # the smallest bf16 number
    x[2] = bf16(1e-36 * x[2])
    x[3] = bf16(1e30 * x[3])
    x[4, 3] = 3.3e38
    x[4] = bf16(x[4])
    x[5] = 0.0
    x[5, cols - 1] = 1.0
    x[6] = (np.arange(cols) % 64) + 0.5                         # codes halfway between two numbers under a largest one of 127
    x[6, 7], x[6, 8] = 127.0, -63.5
    x[7, 1] = np.inf
    x[8, cols - 2] = np.nan
    x[9, 0] = -np.inf
    x[9, 1] = np.inf
    residual = np.zeros_like(x)
    residual[10] = -x[10]                                       # a sum of zeros
    for r in (None, residual):
        got, want = run_norm(torch, x, r, weight, 1e-6), norm_oracle(x, r, weight, 1e-6)
        fine = check_norm(got, want)
        assert fine.tolist() == [True] * 7 + [False] * 3 + [True] * 2
        assert not got[2][7:10].any() and np.isnan(got[1][8]).all()
    assert set(np.abs(got[2][6]) % 2) == {0.0, 1.0} and got[2][6, 0] == 0 and got[2][6, 1] == 2 and got[2][6, 8] == -64
    with pytest.raises(hb.HfxError):
        run_norm(torch, x, None, weight, float("nan"))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [64, 4096])
def test_norm_of_tiny_rows_without_eps(cols):
    """1 / sqrt(mean) past the range of 32 bits; the codes' scale is that of a largest magnitude of 2^-100."""
    import torch
    g = np.random.default_rng(cols)
    x = bf16(g.standard_normal((5, cols)))
    for i, size in enumerate((2.0 ** -126, 2.0 ** -131, 2.0 ** -110, 2.0 ** -99)):
        x[i] = bf16(size * x[i])
    weight = bf16(1.0 + 0.3 * g.standard_normal(cols))
    got, want = run_norm(torch, x, None, weight, 0.0), norm_oracle(x, None, weight, 0.0)
    assert (np.abs(got[1] - want[1]) <= (HALF_BF16 + 3 * 2.0 ** -24) * np.abs(want[1])).all()
    assert np.array_equal(got[2], want[2]) and not got[2][:2].any() and got[2][3:].any()      # (127 2^100 of 2^-110 is an eighth: four of those are a code of 1)


@pytest.mark.gpu
def test_the_most_rows_and_channels():
    import torch
    g, stream, most = torch.Generator(device="cuda").manual_seed(3), torch.cuda.current_stream(), 1 << 21
    x = torch.randn((most, 16), generator=g, device="cuda").bfloat16()
    codes, scales = torch.empty((most, 16), dtype=torch.int8, device="cuda"), torch.empty(most, device="cuda")
    hb.hfx_rms_norm(hb.make_norm(torch.ones(16, dtype=torch.bfloat16, device="cuda"), 0.0), most, x, 16, None, 0, None, None, codes, scales, stream)
    by_norm = codes.clone()
    hb.hfx_quantise_rows(hb.HFX_ACT_NONE, most, 16, x, 16, None, 0, None, codes, scales, stream)
    top = x.float().abs().amax(1, keepdim=True)
    full = torch.full_like(top, 127.0)                          # (a division by a Python number is not one)
    assert torch.equal(codes, torch.round(x.float() * (full / top)).to(torch.int8)) and torch.equal(codes, by_norm) and torch.equal(scales, (top / full)[:, 0])
    for rows, n in ((most, 1), (most, 33), (1, most), (16, most), (33, most)):
        out = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
        hb.hfx_matmul_rows(hb.make_weight_q8(codes[:n], scales[:n]), rows, codes, 16, scales, out, n, False, stream)
        sums = codes[:rows].float() @ codes[:n].float().T           # (exact: no sum passes 2^24)
        assert torch.equal(out, (sums * scales[:rows, None] * scales[None, :n]).bfloat16())
        del out, sums


@pytest.mark.gpu
def test_empty_tensors():
    import torch
    def empty(cols, dtype):
        return torch.empty((0, cols), dtype=dtype, device="cuda")
    codes, scales, stream = empty(64, torch.int8), torch.empty(0, device="cuda"), torch.cuda.current_stream()
    x = empty(64, torch.bfloat16)
    hb.hfx_rms_norm(hb.make_norm(torch.ones(64, dtype=torch.bfloat16, device="cuda"), 0.0), 0, x, 64, x, 64, x, None, codes, scales, stream)
    hb.hfx_quantise_rows(hb.HFX_ACT_SILU, 0, 64, x, 64, None, 0, None, codes, scales, stream)
    weight = hb.make_weight_q8(torch.ones((5, 64), dtype=torch.int8, device="cuda"), torch.ones(5, device="cuda"))
    hb.hfx_matmul_rows(weight, 0, codes, 64, scales, empty(5, torch.float32), 5, True, stream)
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(3, 2048), (2, 40000)])
def test_norm_in_place_and_by_parts(rows, cols):
    """The sum over x or over the residual; results in bf16 alone and in 8 bits alone: the same bits."""
    import torch
    g = np.random.default_rng(5)
    x, residual = device(torch, g.standard_normal((rows, cols))), device(torch, g.standard_normal((rows, cols)))
    norm = hb.make_norm(device(torch, 1.0 + 0.1 * g.standard_normal(cols)), 1e-5)
    stream = torch.cuda.current_stream()

    def call(x, residual, total, want_out, want_codes):
        out = torch.empty_like(x) if want_out else None
        codes, scales = (torch.empty((rows, cols), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")) if want_codes else (None, None)
        hb.hfx_rms_norm(norm, rows, x, cols, residual, cols, total, out, codes, scales, stream)
        torch.cuda.synchronize()
        return total, out, codes, scales
    total, out, codes, scales = call(x, residual, torch.empty_like(x), True, True)
    a, b = x.clone(), residual.clone()
    assert torch.equal(call(a, b, a, True, False)[1], out) and torch.equal(a, total) and torch.equal(b, residual)
    a = x.clone()
    got = call(a, b, b, False, True)
    assert torch.equal(got[2], codes) and torch.equal(got[3], scales) and torch.equal(b, total) and torch.equal(a, x)
    assert torch.equal(call(total, None, None, True, False)[1], out)


# ------------------------------------------------------------------ rows to 8 bits
def run_rows(torch, activation, x, times, extra=0, want_out=True, behind=2):
    rows, cols = x.shape
    dx = strided(torch, device(torch, x), extra)
    dt = None if times is None else strided(torch, device(torch, times), extra)
    out = torch.full((rows + behind, cols), 7.0, dtype=torch.bfloat16, device="cuda") if want_out else None
    codes = torch.full((rows + behind, cols), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((rows + behind,), 7.0, dtype=torch.float32, device="cuda")
    hb.hfx_quantise_rows(activation, rows, cols, dx, cols + extra, dt, cols + extra, out, codes, scales, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for t, was in ((out, 7.0), (codes, 99), (scales, 7.0)):
        assert t is None or bool((t[rows:] == was).all())
    return [None if t is None else t[:rows].cpu().double().numpy() for t in (out, codes, scales)]


SIZES = [(1, 16, 0), (3, 80, 8), (40, 1024, 0), (5, 1376, 8), (2, 8192, 0), (3, 14336, 0), (2, 33008, 8), (1, 131056, 0), (300, 6160, 8), (2100, 4112, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("with_times", [False, True])
@pytest.mark.parametrize("rows,cols,extra", SIZES)
def test_rows_as_they_are(rows, cols, extra, with_times):
    import torch
    g = np.random.default_rng(rows + cols)
    x, times = bf16(g.standard_normal((rows, cols))), bf16(g.standard_normal((rows, cols))) if with_times else None
    v = (x if times is None else x * times).astype(np.float32)          # exact: 8 bits times 8 bits
    codes, top = to_codes(v)
    out, got, scales = run_rows(torch, hb.HFX_ACT_NONE, x, times, extra)
    assert np.array_equal(got, codes)
    assert np.array_equal(scales, (top[:, 0].astype(np.float32) / np.float32(127)).astype(np.float64))
    assert np.array_equal(out, bf16(v))


@pytest.mark.gpu
@pytest.mark.parametrize("with_times", [False, True])
@pytest.mark.parametrize("rows,cols,extra", SIZES)
def test_rows_through_silu(rows, cols, extra, with_times):
    import torch
    g = np.random.default_rng(rows * 7 + cols)
    x, times = bf16(4.0 * g.standard_normal((rows, cols))), bf16(g.standard_normal((rows, cols))) if with_times else None
    x[0, :4] = 90.0, -90.0, 0.0, -1e-30
    v = x / (1.0 + np.exp(-x))
    if times is not None:
        v = v * times
    top = np.abs(v).max(1)
    out, codes, scales = run_rows(torch, hb.HFX_ACT_SILU, x, times, extra)
    assert (np.abs(scales - top / 127.0) <= 2.0 ** -20 * top / 127.0).all()
    assert (np.abs(codes) <= 127).all() and (np.abs(codes).max(1) == 127).all()
    assert (np.abs(codes - v * 127.0 / top[:, None]) <= 0.5 + 1.4e-4).all()
    assert (np.abs(out - v) <= (HALF_BF16 + 2.0 ** -20) * np.abs(v) + 2.0 ** -126).all()
    assert np.array_equal(run_rows(torch, hb.HFX_ACT_SILU, x, times, extra, want_out=False)[1], codes)


@pytest.mark.gpu
@pytest.mark.parametrize("activation", [hb.HFX_ACT_NONE, hb.HFX_ACT_SILU])
def test_rows_that_are_zero_tiny_huge_or_not_finite(activation):
    import torch
    g = np.random.default_rng(2)
    x = bf16(g.standard_normal((8, 1040)))
    x[0] = 0.0
    x[1] = bf16(1e-37 * x[1])                                   # below 2^-100: codes of zero
    x[2] = bf16(np.abs(1e37 * x[2]))
    x[3, 900] = np.inf
    x[4, 2] = np.nan
    x[5] = -np.abs(x[5])
    x[5, 7] = -np.inf                                           # silu of it is not a number
    out, codes, scales = run_rows(torch, activation, x, None)
    assert not codes[[0, 1, 3, 4, 5]].any()
    assert np.isnan(scales[3:6]).all() and np.isfinite(scales[[0, 1, 2, 6, 7]]).all()
    assert scales[0] == scales[1] == float(np.float32(2.0 ** -100) / np.float32(127))
    assert np.abs(codes[2]).max() == 127 and np.abs(codes[6]).max() == 127


@pytest.mark.gpu
def test_rows_in_place():
    import torch
    x, t = device(torch, np.random.default_rng(0).standard_normal((2, 5, 2048)))
    stream = torch.cuda.current_stream()
    want = torch.empty_like(x)
    hb.hfx_quantise_rows(hb.HFX_ACT_SILU, 5, 2048, x, 2048, t, 2048, want, None, None, stream)
    a, b = x.clone(), t.clone()
    hb.hfx_quantise_rows(hb.HFX_ACT_SILU, 5, 2048, a, 2048, t, 2048, a, None, None, stream)
    hb.hfx_quantise_rows(hb.HFX_ACT_SILU, 5, 2048, x, 2048, b, 2048, b, None, None, stream)
    assert torch.equal(a, want) and torch.equal(b, want)


@pytest.mark.gpu
@pytest.mark.parametrize("beside", [90.0, -1000.0, float("inf"), float("nan")])
def test_silu_of_a_value_does_not_depend_on_those_beside_it(beside):
    """One value in 512 far out, or not finite: the results of the others keep their bits."""
    import torch
    rows, cols, stream = 2048, 4096, torch.cuda.current_stream()
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.empty((rows, cols), device="cuda").normal_(0.0, 16.0, generator=gen).clamp_(-80.0, 80.0).bfloat16()
    times = torch.empty((rows, cols), device="cuda").normal_(generator=gen).bfloat16()
    outs = []
    for value in (0.0, beside):
        x[:, 77::512] = value
        outs.append(torch.empty_like(x))
        hb.hfx_quantise_rows(hb.HFX_ACT_SILU, rows, cols, x, cols, times, cols, outs[-1], None, None, stream)
        outs[-1][:, 77::512] = 0.0
    assert int((outs[0].view(torch.int16) != outs[1].view(torch.int16)).sum()) == 0


@pytest.mark.gpu
def test_silu_of_every_number():
    """One number to a row, so that its result is seen through the scale, times 2^60 where it is small.  The value 2^-21, as above; the scale's division 2^-24."""
    import torch
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[torch.isfinite(x)]
    for part, up in ((x.abs() <= 1.0, 2.0 ** 60), ((x.abs() > 1.0) & (x.abs() <= 80.0), 2.0 ** 60), ((x.abs() > 80.0) & (x.abs() <= 110.0), 2.0 ** 60), (x.abs() > 110.0, 1.0)):
        n = int(part.sum())
        rows = torch.zeros((n, 16), dtype=torch.bfloat16, device="cuda")
        rows[:, 3] = x[part].cuda()
        out, codes, scales = torch.empty_like(rows), torch.empty((n, 16), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        hb.hfx_quantise_rows(hb.HFX_ACT_SILU, n, 16, rows, 16, torch.full_like(rows, up), 16, out, codes, scales, torch.cuda.current_stream())
        v = x[part].double().numpy()
        with np.errstate(over="ignore"):
            v = v / (1.0 + np.exp(-v))
        top = np.maximum(np.abs(v) * up, 2.0 ** -100)
        # (results below 2^-126 are whole numbers of 2^-149, before the product with `up`: half of one)
        assert (np.abs(scales.cpu().double().numpy() * 127.0 - top) <= (2.0 ** -21 + 2.0 ** -24) * top + 2.0 ** -150 * up).all()
        far = v * up
        assert (np.abs(out[:, 3].cpu().double().numpy() - far) <= (HALF_BF16 + 2.0 ** -20) * np.abs(far) + 2.0 ** -150 * up + 2.0 ** -133).all()


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [4112, 8192])
def test_a_row_does_not_depend_on_the_number_of_rows(cols):
    import torch
    stream = torch.cuda.current_stream()
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, times = torch.empty((2, 700, cols), device="cuda").normal_(0.0, 3.0, generator=gen).bfloat16()
    x[:, 9::700] = 100.0
    norm = hb.make_norm(times[0], 1e-6)

    def call(rows):
        codes, scales = torch.empty((2, rows, cols), dtype=torch.int8, device="cuda"), torch.empty((2, rows), device="cuda")
        total = torch.empty_like(x[:rows])
        hb.hfx_quantise_rows(hb.HFX_ACT_SILU, rows, cols, x, cols, times, cols, None, codes[0], scales[0], stream)
        hb.hfx_rms_norm(norm, rows, x, cols, times, cols, total, None, codes[1], scales[1], stream)
        return codes, scales
    codes, scales = call(700)
    for rows in (1, 256, 257):
        few_codes, few_scales = call(rows)
        assert torch.equal(few_codes, codes[:, :rows]) and torch.equal(few_scales, scales[:, :rows])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(9601, 512), (4801, 1024), (2407, 2048), (1203, 4096)])
def test_rows_past_the_caches(rows, cols):
    """Calls of more than 32 MB of each thread count: the same bits as in calls of a tenth of the rows."""
    import torch
    stream = torch.cuda.current_stream()
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, y = torch.empty((2, rows, cols), device="cuda").normal_(0.0, 2.0, generator=gen).bfloat16()
    norm = hb.make_norm(y[0] + 1.0, 1e-6)

    def call(first, count):
        total, out, normed = torch.empty((3, count, cols), dtype=torch.bfloat16, device="cuda")
        codes, scales = torch.empty((2, count, cols), dtype=torch.int8, device="cuda"), torch.empty((2, count), device="cuda")
        hb.hfx_rms_norm(norm, count, x[first:], cols, y[first:], cols, total, normed, codes[0], scales[0], stream)
        hb.hfx_quantise_rows(hb.HFX_ACT_SILU, count, cols, x[first:], cols, y[first:], cols, out, codes[1], scales[1], stream)
        return total, out, normed, *codes, *scales
    whole, part = call(0, rows), -(-rows // 10)
    parts = [call(first, min(part, rows - first)) for first in range(0, rows, part)]
    for i, got in enumerate(whole):
        assert torch.equal(got, torch.cat([p[i] for p in parts])), i
    assert torch.equal(whole[0], (x.float() + y.float()).bfloat16())


# ------------------------------------------------------------------ products
def product_oracle(codes, scales, weight, weight_scales, bias, fp32):
    """With the operator's roundings; the sums by a product in 64 bits, which holds them exactly."""
    y = (codes.astype(np.float64) @ weight.astype(np.float64).T).astype(np.float32)
    with np.errstate(invalid="ignore"):
        y = y * scales[:, None] * weight_scales[None]
    if bias is not None:
        y = y + bias.astype(np.float32)
    return y.astype(np.float64) if fp32 else bf16(y)


def run_product(torch, codes, scales, weight, weight_scales, bias, fp32, extra=(0, 0, 0), behind=3):
    """extra: elements between the rows of codes, weight and results."""
    rows, k = codes.shape
    n = len(weight)
    dc, dw = strided(torch, device(torch, codes, torch.int8), extra[0]), strided(torch, device(torch, weight, torch.int8), extra[1])
    handle = hb.make_weight_q8(dw[:, :k], device(torch, weight_scales, torch.float32), None if bias is None else device(torch, bias))
    out = torch.full((rows + behind, n + extra[2]), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
    hb.hfx_matmul_rows(handle, rows, dc, k + extra[0], device(torch, scales, torch.float32), out, n + extra[2], fp32, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert bool((out[rows:] == 7.0).all()) and bool((out[:, n:] == 7.0).all())
    return out[:rows, :n].cpu().double().numpy()


def product_inputs(g, rows, n, k, with_bias):
    codes, weight = g.integers(-128, 128, (rows, k)).astype(np.int8), g.integers(-128, 128, (n, k)).astype(np.int8)
    scales, weight_scales = (np.exp(g.standard_normal(m)).astype(np.float32) / np.float32(70.0 * k ** 0.25) for m in (rows, n))
    return codes, scales, weight, weight_scales, bf16(g.standard_normal(n)) if with_bias else None


def check_product(torch, rows, n, k, with_bias, fp32, extra=(0, 0, 0), seed=0):
    a = product_inputs(np.random.default_rng([rows, n, k, seed]), rows, n, k, with_bias)
    got, want = run_product(torch, *a, fp32, extra), product_oracle(*a, fp32)
    wrong = np.argwhere(got != want)
    assert not len(wrong), (rows, n, k, len(wrong), wrong[:4].tolist(), got[tuple(wrong[0])], want[tuple(wrong[0])])


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 32, 33, 48, 63, 64, 65, 96, 128, 129, 200, 256, 257, 520, 1030])
def test_products_of_any_number_of_rows(rows):
    import torch
    for n, k, fp32 in ((640, 512, False), (1000, 1040, True), (37, 2064, False)):
        check_product(torch, rows, n, k, rows % 2 == 0, fp32)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 3, 15, 16, 17, 31, 33, 63, 65, 127, 128, 129, 255, 257, 1001])
def test_products_of_any_number_of_channels(n):
    import torch
    for rows, k, fp32 in ((1, 256, True), (20, 144, False), (70, 400, True), (300, 256, False)):
        check_product(torch, rows, n, k, n % 2 == 1, fp32)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [16, 32, 48, 64, 80, 112, 128, 144, 240, 256, 272, 384, 496, 768, 1008, 4096, 4112])
def test_products_over_any_length(k):
    import torch
    for rows, n, fp32 in ((1, 70, False), (16, 130, True), (50, 300, False), (150, 270, False), (400, 515, True)):
        check_product(torch, rows, n, k, False, fp32)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,k,extra", [(5, 300, 528, (16, 32, 1)), (33, 64, 256, (48, 0, 8)), (130, 257, 1040, (16, 16, 7)), (700, 768, 640, (0, 64, 128)), (64, 4096, 64, (4080, 16, 3)),
                                            (64, 4090, 8080, (0, 112, 0)), (100, 8200, 4000, (16, 96, 1)), (24, 8200, 4096, (0, 0, 0)), (7, 16400, 272, (0, 3824, 0)), (40, 8200, 144, (0, 3952, 8))])
def test_products_of_rows_that_lie_apart(rows, n, k, extra):
    import torch
    for fp32 in (False, True):
        check_product(torch, rows, n, k, True, fp32, extra)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("n,k", [(4096, 4096), (1280, 8192), (5001, 2048)])
def test_products_of_a_layers_size(rows, n, k):
    import torch
    check_product(torch, rows, n, k, True, False)


# Sizes at which the tiles of every kernel come up, with parts of tiles at both edges, sums of one stage and up, whole and not, one tile to a workgroup and several.
FILLING = [(771, 8208, 4099), (1491, 4112, 4100), (4100, 400, 4100), (4100, 384, 4100), (3000, 144, 3000), (3000, 784, 6100), (2047, 1040, 16390), (5000, 512, 5000), (5000, 384, 5003),
           (5000, 272, 5000), (1500, 1040, 8200), (8219, 256, 6147), (8219, 528, 6147), (777, 1024, 8192), (1000, 2000, 1500), (2050, 400, 9000), (600, 512, 12000), (1030, 512, 9001),
           (6000, 16, 7001), (2000, 128, 5000), (4096, 1024, 4096), (520, 8192, 4096), (3100, 2064, 2050),
           (1324, 272, 9280), (2471, 416, 4910), (929, 3856, 6111), (4654, 400, 10263), (665, 4384, 9861), (639, 3984, 6414), (1043, 3984, 2648), (4255, 3984, 877), (3345, 1504, 4599),
           (4543, 16, 6456), (3153, 16, 7319), (1039, 16, 2186), (4410, 272, 208), (567, 144, 394),
           (64, 4112, 6144), (37, 4240, 6001), (128, 496, 4000), (33, 16, 6144), (60, 144, 6144), (100, 272, 4000), (64, 8336, 4090), (24, 8208, 4097), (128, 4128, 6144),
           (4128, 1024, 16384), (6200, 1040, 9001), (8224, 1040, 8203), (4500, 1040, 8200), (4128, 2064, 16387), (4100, 1024, 16384), (4104, 4112, 4100),
           (250, 4112, 6100), (200, 4240, 6144), (500, 8208, 4090), (400, 144, 4000), (1000, 400, 3900), (900, 656, 2500), (130, 528, 16001)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,k,n", FILLING)
def test_products_that_fill_the_chip(rows, k, n):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows + n)
    codes, weight = (torch.randint(-128, 128, (m, k), dtype=torch.int8, device="cuda", generator=gen) for m in (rows, n))
    scales, weight_scales = (torch.rand(m, device="cuda", generator=gen) + 0.01 for m in (rows, n))
    bias = torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1000.0, generator=gen)
    sums = (codes.double() @ weight.double().T).float()         # exact in 64 bits, rounded once
    for fp32, with_bias in ((False, False), (True, False), (False, True)):
        want = sums * scales[:, None] * weight_scales
        if with_bias:
            want = want + bias.float()
        out = torch.full((rows + 2, n), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
        hb.hfx_matmul_rows(hb.make_weight_q8(weight, weight_scales, bias if with_bias else None), rows, codes, k, scales, out, n, fp32, torch.cuda.current_stream())
        assert bool((out[rows:] == 7.0).all())
        assert torch.equal(out[:rows], want.to(out.dtype))


# (rows, k, elements from one of the weight's rows to the next, n): tiles that take the stages of the sum in turns, whole chips of them and several layers, with whole and partial
# stages and only those; the few rows that the kernel for them takes, and one more.
APART = [(64, 4096, 4096, 16384), (33, 4096, 4096, 16383), (50, 4016, 4096, 16384), (48, 272, 4096, 16370), (40, 112, 4096, 16384), (64, 1168, 8192, 16333), (64, 8192, 8192, 4096), (40, 2000, 4096, 4090),
         (17, 4096, 4096, 8200), (100, 384, 4096, 4096), (1, 8192, 8192, 4096), (7, 512, 512, 640), (8, 512, 512, 640), (9, 512, 512, 640), (8, 4112, 4128, 4099), (8, 8208, 8208, 2050), (9, 4096, 4096, 4096),
         (100, 4096, 4096, 8190), (150, 1040, 1040, 4096), (200, 400, 416, 4090), (128, 2064, 2064, 6100)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,k,stride,n", APART)
def test_products_of_few_rows_and_many_channels(rows, k, stride, n):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows + n + k)
    codes, weight = (torch.randint(-128, 128, (m, k), dtype=torch.int8, device="cuda", generator=gen) for m in (rows, n))
    weight = strided(torch, weight, stride - k)[:, :k]
    scales, weight_scales = (torch.rand(m, device="cuda", generator=gen) + 0.01 for m in (rows, n))
    bias = torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1000.0, generator=gen)
    sums = (codes.double() @ weight.double().T).float()         # exact in 64 bits, rounded once
    for fp32 in (False, True):
        for with_bias in (False, True):
            want = sums * scales[:, None] * weight_scales
            if with_bias:
                want = want + bias.float()
            out = torch.full((rows + 2, n + 3), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
            hb.hfx_matmul_rows(hb.make_weight_q8(weight, weight_scales, bias if with_bias else None), rows, codes, k, scales, out, n + 3, fp32, torch.cuda.current_stream())
            assert bool((out[rows:] == 7.0).all()) and bool((out[:, n:] == 7.0).all())
            assert torch.equal(out[:rows, :n], want.to(out.dtype))


def test_every_kernel_is_reached():
    """The sizes of the two tests above come to every kernel that a product can take, with the stages of the sum in order and, where there is such a form, in turns."""
    choose, ways = hb.load().hfx_internal_matmul_ways, (ctypes.c_int * 2)()
    choose.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int64, ctypes.POINTER(ctypes.c_int)]
    reached = {}
    for rows, k, stride, n in [(rows, k, k, n) for rows, k, n in FILLING] + APART:
        launches = choose(rows, n, k, stride, ways)
        assert launches in (1, 2)
        for way in ways[:launches]:
            reached.setdefault(way, []).append((rows, k, stride, n))
    ways_there_are = choose(0, 0, 0, 0, ways)
    assert set(range(ways_there_are)) <= set(reached), sorted(set(range(ways_there_are)) - set(reached))
    assert {101, 103} == {way for way in reached if way >= 100}                          # 32 by 32 and 64 by 64
    assert all(len(sizes) >= 3 for sizes in reached.values()), {way: sizes for way, sizes in reached.items() if len(sizes) < 3}
    assert {choose(rows, 640, 512, 512, ways) and ways[0] for rows in (1, 7, 8)} == {0} and choose(9, 640, 512, 512, ways) == 1 and ways[0] == 1


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n", [(1, 260), (30, 260), (80, 260), (260, 260), (700, 4100)])
def test_the_longest_sums(rows, n):
    """All codes -128 over the longest row: 2^31 - 2^18, the largest sum there is; and the smallest."""
    import torch
    k = 131056
    codes, weight = np.full((rows, k), -128, np.int8), np.full((n, k), -128, np.int8)
    weight[1::2] = 127
    one = np.ones(rows, np.float32), np.ones(n, np.float32)
    got = run_product(torch, codes, one[0], weight, one[1], None, True)
    assert (got[:, 0::2] == float(np.float32(128 * 128 * k))).all() and (got[:, 1::2] == float(np.float32(-128 * 127 * k))).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 40, 270])
def test_scales_that_are_not_numbers_stay_in_their_row_and_channel(rows):
    import torch
    a = list(product_inputs(np.random.default_rng(rows), rows, 300, 256, False))
    a[1][rows // 2], a[3][17] = np.nan, np.nan
    got, want = run_product(torch, *a, False), product_oracle(*a, False)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got).sum() == rows + 300 - 1


@pytest.mark.gpu
def test_products_past_4_gb():
    """Weights, rows and results whose offsets pass 32 bits: their last parts against the same parts alone."""
    import torch
    stream = torch.cuda.current_stream()
    gen = torch.Generator(device="cuda").manual_seed(3)

    def codes(*shape):
        return torch.randint(-128, 128, shape, dtype=torch.int8, device="cuda", generator=gen)
    for rows, n, k, w_stride, c_stride in ((70, 70000, 64, 65536, 64), (70000, 70, 64, 64, 65536), (50000, 50000, 64, 64, 64)):
        w = torch.zeros((n, w_stride), dtype=torch.int8, device="cuda")
        c = torch.zeros((rows, c_stride), dtype=torch.int8, device="cuda")
        w[:, :k], c[:, :k] = codes(n, k), codes(rows, k)
        ws, cs = torch.rand(n, device="cuda", generator=gen), torch.rand(rows, device="cuda", generator=gen)
        out = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
        assert max(w.numel(), c.numel(), 2 * out.numel()) > 1 << 32
        hb.hfx_matmul_rows(hb.make_weight_q8(w[:, :k], ws), rows, c, c_stride, cs, out, n, False, stream)
        for r, j in ((slice(rows - 65, rows), slice(n - 65, n)), (slice(0, 33), slice(n - 33, n)), (slice(rows - 33, rows), slice(0, 70))):
            y = (c[r, :k].double() @ w[j, :k].double().T).float() * cs[r, None] * ws[j]
            assert torch.equal(out[r, j], y.to(torch.bfloat16))
        del w, c, out


@pytest.mark.gpu
def test_a_layers_calls_on_a_stream_and_in_a_graph():
    """Norm, projection, activation, projection: eager, on another stream, and captured; the graph's inputs change between its replays."""
    import torch
    rows, hidden, wide = 37, 1024, 1792
    gen = torch.Generator(device="cuda").manual_seed(1)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    norm = hb.make_norm(normal(hidden), 1e-6)

    def weight(n, k):
        codes, scales = torch.empty((n, k), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        hb.hfx_quantise_rows(hb.HFX_ACT_NONE, n, k, normal(n, k) * k ** -0.5, k, None, 0, None, codes, scales, torch.cuda.current_stream())
        return hb.make_weight_q8(codes, scales)
    up, down = weight(2 * wide, hidden), weight(hidden, wide)
    x, residual = normal(rows, hidden), normal(rows, hidden)

    def buffers():
        return dict(sum=torch.empty_like(x), c1=torch.empty((rows, hidden), dtype=torch.int8, device="cuda"), s1=torch.empty(rows, device="cuda"),
                    both=torch.empty((rows, 2 * wide), dtype=torch.bfloat16, device="cuda"), c2=torch.empty((rows, wide), dtype=torch.int8, device="cuda"),
                    s2=torch.empty(rows, device="cuda"), out=torch.empty_like(x))

    def layer(b, stream):
        hb.hfx_rms_norm(norm, rows, x, hidden, residual, hidden, b["sum"], None, b["c1"], b["s1"], stream)
        hb.hfx_matmul_rows(up, rows, b["c1"], hidden, b["s1"], b["both"], 2 * wide, False, stream)
        hb.hfx_quantise_rows(hb.HFX_ACT_SILU, rows, wide, b["both"], 2 * wide, b["both"][:, wide:], 2 * wide, None, b["c2"], b["s2"], stream)
        hb.hfx_matmul_rows(down, rows, b["c2"], wide, b["s2"], b["out"], hidden, False, stream)
    eager, other, captured = buffers(), buffers(), buffers()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        layer(other, side)
    layer(eager, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert all(torch.equal(eager[n], other[n]) for n in eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer(captured, torch.cuda.current_stream())
    for turn in range(4):
        x.normal_(generator=gen)
        residual.mul_(0.5 + turn)
        layer(eager, torch.cuda.current_stream())
        torch.cuda.synchronize()
        for b in captured.values():
            b.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(eager[n], captured[n]) for n in eager)
        assert bool(torch.isfinite(eager["out"]).all()) and float(eager["out"].float().std()) > 0.01


@pytest.mark.gpu
def test_calls_on_two_streams_at_once_and_a_product_of_two_launches_in_a_graph():
    """Nothing that calls share: each stream's results are those of its calls alone, also while a graph of a product that takes two launches is replayed."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(17)

    def random_codes(rows, k):
        return torch.randint(-127, 128, (rows, k), dtype=torch.int8, device="cuda", generator=gen), torch.rand(rows, device="cuda", generator=gen) + 0.1
    rows, n, k = 4128, 16384, 1024
    large, (large_codes, large_scales) = hb.make_weight_q8(*random_codes(n, k)), random_codes(rows, k)
    small, norm = hb.make_weight_q8(*random_codes(900, 2048)), hb.make_norm(torch.rand(2048, generator=gen, device="cuda").bfloat16(), 1e-6)
    x = torch.randn((50, 2048), generator=gen, device="cuda").bfloat16()
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [torch.empty((rows, n), dtype=torch.bfloat16, device="cuda") for _ in range(3)]

    def chain(stream):
        with torch.cuda.stream(stream):
            codes, scales, out = torch.empty((50, 2048), dtype=torch.int8, device="cuda"), torch.empty(50, device="cuda"), torch.empty((50, 900), device="cuda")
        hb.hfx_rms_norm(norm, 50, x, 2048, None, 0, None, None, codes, scales, stream)
        hb.hfx_matmul_rows(small, 50, codes, 2048, scales, out, 900, True, stream)
        return out
    want = chain(torch.cuda.current_stream())
    hb.hfx_matmul_rows(large, rows, large_codes, k, large_scales, outs[0], n, False, torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=first):
        hb.hfx_matmul_rows(large, rows, large_codes, k, large_scales, outs[1], n, False, torch.cuda.current_stream())
    for turn in range(3):
        outs[1].zero_()
        outs[2].zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(first):
            graph.replay()
        got = [chain(second) for _ in range(8)]
        hb.hfx_matmul_rows(large, rows, large_codes, k, large_scales, outs[2], n, False, second)
        got += [chain(first), chain(second)]
        torch.cuda.synchronize()
        assert torch.equal(outs[1], outs[0]) and torch.equal(outs[2], outs[0]) and all(torch.equal(o, want) for o in got)


# ------------------------------------------------------------------ refusals, on the host
class Fake:
    """A norm or weight without memory: its numbers are addresses."""

    def __init__(self, kind, *args):
        self.held = kind(*args)
        self.address = self.held.address


def refused(call, code):
    with pytest.raises(hb.HfxError) as e:
        call()
    assert e.value.code == code


def test_what_the_norm_refuses():
    ok = dict(norm=(16, 64, 1e-6), rows=2, x=32, x_stride=64, residual=None, residual_stride=0, sum=None, out=48, codes=None, scales=None)

    def call(**change):
        a = {**ok, **change}
        norm = a.pop("norm")
        hb.hfx_rms_norm(Fake(hb.hfx_norm, *norm) if norm else None, *a.values())
    call(rows=0)                                                # nothing to do
    call(rows=0, residual=64, residual_stride=64, sum=32, codes=64, scales=4)
    call(rows=0, x=None, out=None)
    for change in (dict(norm=None), dict(norm=(None, 64, 1e-6)), dict(x=None), dict(residual=16), dict(sum=16), dict(out=None), dict(codes=16), dict(scales=16), dict(out=None, codes=16)):
        refused(lambda: call(**change), hb.HFX_ERR_NULL)
    for change in (dict(rows=-1), dict(rows=(1 << 21) + 1), dict(norm=(16, 0, 1e-6)), dict(norm=(16, 72, 1e-6), x_stride=72), dict(norm=(16, 131072, 1e-6), x_stride=131072), dict(norm=(16, -16, 1e-6)),
                   dict(norm=(16, 64, -1.0)), dict(norm=(16, 64, float("nan"))), dict(norm=(16, 64, float("inf"))), dict(x_stride=56), dict(x_stride=-64),
                   dict(x_stride=(1 << 22) + 8), dict(residual=16, sum=64, residual_stride=63), dict(residual=16, residual_stride=64, sum=32, x_stride=72),
                   dict(residual=16, residual_stride=72, sum=16)):
        refused(lambda: call(**change), hb.HFX_ERR_SHAPE)
    for change in (dict(x=24), dict(norm=(8, 64, 1e-6)), dict(out=40), dict(x_stride=68), dict(residual=18, sum=64, residual_stride=64), dict(residual=16, sum=72, residual_stride=64),
                   dict(residual=16, sum=64, residual_stride=70), dict(codes=8, scales=4), dict(codes=16, scales=2)):
        refused(lambda: call(**change), hb.HFX_ERR_ALIGN)


def test_what_the_rows_to_8_bits_refuse():
    ok = dict(activation=hb.HFX_ACT_SILU, rows=2, cols=64, x=32, x_stride=64, times=None, times_stride=0, out=None, codes=48, scales=4)

    def call(**change):
        hb.hfx_quantise_rows(*{**ok, **change}.values())
    call(rows=0)
    call(rows=0, times=64, times_stride=128)
    call(rows=0, x=None, codes=None, scales=None)
    for change in (dict(x=None), dict(codes=None), dict(scales=None), dict(codes=None, scales=None)):
        refused(lambda: call(**change), hb.HFX_ERR_NULL)
    for change in (dict(activation=2), dict(activation=-1), dict(rows=-3), dict(cols=8), dict(cols=24), dict(cols=131072, x_stride=131072), dict(x_stride=63), dict(times=16, times_stride=0),
                   dict(times=16, times_stride=(1 << 22) + 16), dict(out=32), dict(times=16, times_stride=64, out=16), dict(out=32, codes=None, scales=None, x_stride=72),
                   dict(times=16, times_stride=72, out=16, codes=None, scales=None)):
        refused(lambda: call(**change), hb.HFX_ERR_SHAPE)
    for change in (dict(x=40), dict(times=40, times_stride=64), dict(times=32, times_stride=68), dict(out=8), dict(codes=50), dict(scales=6), dict(x_stride=66)):
        refused(lambda: call(**change), hb.HFX_ERR_ALIGN)


def test_what_the_products_refuse():
    good = dict(codes=16, scales=4, bias=None, n=32, k=64, stride=64)
    ok = dict(weight={}, rows=2, codes=32, codes_stride=64, scales=8, out=48, out_stride=32, fp32=False)

    def call(**change):
        a = {**ok, **change}
        weight = a.pop("weight")
        hb.hfx_matmul_rows(None if weight is None else Fake(hb.hfx_weight_q8, *{**good, **weight}.values()), *a.values())
    call(rows=0)
    call(rows=0, codes=None, scales=None, out=None)
    for change in (dict(weight=None), dict(weight=dict(codes=None)), dict(weight=dict(scales=None)), dict(codes=None), dict(scales=None), dict(out=None)):
        refused(lambda: call(**change), hb.HFX_ERR_NULL)
    for change in (dict(rows=-1), dict(rows=(1 << 21) + 1), dict(weight=dict(n=0)), dict(weight=dict(n=(1 << 21) + 1), out_stride=1 << 22), dict(weight=dict(k=0)), dict(weight=dict(k=56)),
                   dict(weight=dict(k=131072, stride=131072), codes_stride=131072), dict(weight=dict(stride=48)), dict(weight=dict(stride=1 << 23)), dict(codes_stride=48), dict(codes_stride=-64),
                   dict(out_stride=31), dict(out_stride=1 << 23), dict(fp32=2), dict(rows=1 << 21, weight=dict(n=1 << 18), out_stride=1 << 18)):
        refused(lambda: call(**change), hb.HFX_ERR_SHAPE)
    for change in (dict(weight=dict(codes=24)), dict(weight=dict(scales=6)), dict(weight=dict(bias=5)), dict(weight=dict(stride=72)), dict(codes=40), dict(codes_stride=72), dict(scales=2), dict(out=24)):
        refused(lambda: call(**change), hb.HFX_ERR_ALIGN)


def test_handles_refuse_other_tensors():
    import torch
    for weight in (torch.zeros(64), torch.zeros(64, dtype=torch.float16), torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(128, dtype=torch.bfloat16)[::2],
                   torch.zeros(64, dtype=torch.bfloat16)):                                   # (the last: in host memory)
        with pytest.raises(ValueError):
            hb.make_norm(weight, 1e-6)
    codes, scales, bias = torch.zeros((8, 64), dtype=torch.int8), torch.zeros(8), torch.zeros(8, dtype=torch.bfloat16)
    for args in ((codes[0], scales), (codes.float(), scales), (codes.T, scales), (codes, scales[:7]), (codes, scales.double()), (codes, torch.zeros(16)[::2]), (codes, scales, bias[:3]),
                 (codes, scales, bias.float()), (codes, scales, bias)):
        with pytest.raises(ValueError):
            hb.make_weight_q8(*args)
