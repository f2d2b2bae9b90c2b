"""The dense operators on the GPU against plain 64-bit references, with bounds from the operations' own rounding."""
import math

import numpy as np
import pytest
import torch

import paper_2404_03019_amd as geot
from paper_2404_03019_amd import autograd as ga

import dense_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = (F32, BF16, F16)
SEED, OFFSET = 0x123456789ABCDEF1, (5 << 32) + 9


def rand(gen, *shape, dtype=F32, scale=1.0, pad=0):
    t = (torch.randn((*shape[:-1], shape[-1] + pad), generator=gen, device=DEV) * scale).to(dtype)
    return t[..., :shape[-1]]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def mask_of(rows, F, p, seed=SEED, offset=OFFSET):
    if p == 1.0:
        return torch.zeros(rows, F, dtype=torch.float64, device=DEV)
    return torch.from_numpy(ref.kept(rows, F, p, seed, offset)).to(DEV).double() / (1.0 - p)


# ---- dropout ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, F, pad", [(1, 1, 0), (1, 7, 0), (3, 8, 0), (65, 4, 1), (7, 100, 0), (130, 47, 2), (257, 128, 8),
                                          (2, 1030, 3), (1, 100_003, 0), (5000, 3, 0)])
@pytest.mark.parametrize("p, residual", [(0.5, False), (0.1, True), (0.0, True), (1.0, True)])
def test_dropout(dtype, rows, F, pad, p, residual):
    g = gen(rows * F)
    x, res = rand(g, rows, F, dtype=dtype, pad=pad), rand(g, rows, F, dtype=dtype, pad=1) if residual else None
    got = geot.dropout(x, p, SEED, OFFSET, residual=res)
    m = mask_of(rows, F, p) if p else torch.ones_like(x, dtype=torch.float64)
    term = m * x.double()
    want = term + (res.double() if residual else 0.0)
    # scale, product and sum in 32 bits
    ref.check(got, want, 3 * ref.U * (term.abs() + want.abs()), "dropout")
    dropped = m == 0
    assert torch.equal(got[dropped], (res if residual else torch.zeros_like(x))[dropped])
    # the gradient: the same mask on another tensor, also through autograd, and no residual in it
    leaf, side = x.clone().requires_grad_(True), res.clone().requires_grad_(True) if residual else None
    up = rand(g, rows, F, dtype=dtype)
    ga.dropout(leaf, p, SEED, OFFSET, residual=side).backward(up)
    ref.check(leaf.grad, m * up.double(), 3 * ref.U * (m * up.double()).abs(), "gradient")
    if residual:
        assert torch.equal(side.grad, up)


def test_dropout_rate_and_independence():
    """A mask keeps 1 - p of its elements to six standard deviations, and masks of other offsets, seeds or rows agree as
    often as independent ones."""
    n, p = 1 << 22, 0.3
    x = torch.ones(1024, n // 1024, device=DEV)
    masks = [geot.dropout(x, p, s, o) != 0 for s, o in ((1, 0), (1, 1), (2, 0), (1 + (1 << 32), 0), (1, 1 << 32))]
    sd = math.sqrt(n * p * (1 - p))
    for m in masks:
        assert abs(int(m.sum()) - n * (1 - p)) <= 6 * sd
    same = p * p + (1 - p) ** 2
    for i in range(len(masks)):
        for j in range(i):
            assert abs(int((masks[i] == masks[j]).sum()) - n * same) <= 6 * math.sqrt(n * same * (1 - same))
    a = masks[0]
    assert abs(int((a[1:] == a[:-1]).sum()) - (n - n // 1024) * same) <= 6 * math.sqrt(n * same * (1 - same))


def test_dropout_mask_is_of_the_place_alone():
    """Columns, types, strides, in-place calls and one-dimensional tensors see the same mask."""
    x = torch.ones(33, 90, device=DEV)
    full = geot.dropout(x, 0.5, SEED, 3) != 0
    for F in (1, 13, 64):
        assert torch.equal(geot.dropout(x[:, :F], 0.5, SEED, 3) != 0, full[:, :F])
    for t in (BF16, F16):
        assert torch.equal(geot.dropout(x.to(t), 0.5, SEED, 3) != 0, full)
    y = x.clone()
    assert geot.dropout(y, 0.5, SEED, 3, out=y) is y and torch.equal(y != 0, full)
    assert torch.equal(geot.dropout(x[0], 0.5, SEED, 3) != 0, full[0])
    w = torch.ones(90, device=DEV)
    assert torch.equal(geot.dropout(w, 0.5, SEED, 3, residual=w) == 1, ~full[0])
    r = x.clone()
    geot.dropout(x, 0.5, SEED, 3, residual=r, out=r)
    assert torch.equal(r == 1, ~full)


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_of_infinities(dtype):
    """What is dropped leaves no trace, whatever it was; what is kept keeps its class."""
    x = torch.tensor([math.inf, -math.inf, math.nan, 1.0] * 64, device=DEV, dtype=dtype).view(4, 64)
    got = geot.dropout(x, 0.5, SEED, 1)
    m = mask_of(4, 64, 0.5, SEED, 1) > 0
    assert torch.equal(got[~m], torch.zeros_like(got[~m])) and torch.equal(torch.isnan(got[m]), torch.isnan(x[m]))
    assert torch.equal(torch.isinf(got[m]), torch.isinf(x[m]))


def test_dropout_past_32_bits():
    """More than 2^32 elements: the last rows see their own mask."""
    rows, F = (1 << 22) + 5, 1032
    x = torch.ones(rows, F, dtype=BF16, device=DEV)
    geot.dropout(x, 0.25, SEED, OFFSET, out=x)
    for first in (0, rows - 3):
        m = torch.from_numpy(ref.kept(3, F, 0.25, SEED, OFFSET, first_row=first)).to(DEV)
        assert torch.equal(x[first:first + 3] != 0, m)


def test_dropout_of_a_long_vector():
    """A vector (edge weights) of more than 2^31 elements: the last columns see their own words."""
    n = (1 << 31) + 4 * 7 + 1
    x = torch.ones(n, dtype=BF16, device=DEV)
    geot.dropout(x, 0.25, SEED, OFFSET, out=x)
    at = (n - 100) // 4
    m = torch.from_numpy(ref.kept(1, n - 4 * at, 0.25, SEED, OFFSET, first_group=at)).to(DEV)[0]
    assert torch.equal(x[4 * at:] != 0, m)


# ---- the gated block -------------------------------------------------------
SHAPES = [(1, 1, 1), (1, 64, 8), (1, 2056, 520), (2, 7, 3), (5, 100, 65), (17, 64, 16), (33, 129, 200), (64, 8, 128), (130, 72, 130),
          (300, 520, 64), (1000, 33, 47), (16, 1500, 300)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M, K, N", SHAPES)
@pytest.mark.parametrize("act, bias, p, pad", [("silu", True, 0.0, 0), ("gelu", False, 0.25, 0), ("relu", True, 0.5, 3),
                                               ("sigmoid", False, 0.0, 8), ("none", True, 0.0, 1)])
def test_gated(dtype, M, K, N, act, bias, p, pad):
    g = gen(M * 1000003 + K * 1009 + N)
    x = rand(g, M, K, dtype=dtype, pad=pad)
    wg, wu = (rand(g, N, K, dtype=dtype, scale=1 / math.sqrt(K), pad=pad) for _ in range(2))
    bg, bu = (rand(g, N, dtype=dtype) if bias else None for _ in range(2))
    grad = rand(g, M, N, dtype=dtype, pad=pad)
    mask = mask_of(M, N, p) if p else None
    want = ref.gated64(x, wg, wu, bg, bu, act, mask, grad)
    out = geot.gated_linear(x, wg, wu, bg, bu, act, p, SEED, OFFSET)
    ref.check(out, *want[0], "out")
    got = geot.gated_linear_backward(grad, x, wg, wu, bg, bu, act, p, SEED, OFFSET)
    for name, t, w in zip(("grad_x", "grad_w_gate", "grad_w_up", "grad_b_gate", "grad_b_up"), got, want[1:]):
        assert (t is None) == (not bias and name.startswith("grad_b"))
        if t is not None:
            ref.check(t, *w, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M, K, N", [(2050, 136, 300), (40_003, 24, 40), (700, 1032, 1100)])
def test_gated_larger(dtype, M, K, N):
    """Several tiles each way, long sums over the rows, and (past one tile a CU) the large tiles."""
    g = gen(5)
    x, wg, wu = rand(g, M, K, dtype=dtype), rand(g, N, K, dtype=dtype, scale=0.1), rand(g, N, K, dtype=dtype, scale=0.1)
    bg, bu, grad = rand(g, N, dtype=dtype), rand(g, N, dtype=dtype), rand(g, M, N, dtype=dtype)
    want = ref.gated64(x, wg, wu, bg, bu, "silu", None, grad)
    ref.check(geot.gated_linear(x, wg, wu, bg, bu), *want[0], "out")
    for i, (t, w) in enumerate(zip(geot.gated_linear_backward(grad, x, wg, wu, bg, bu), want[1:])):
        ref.check(t, *w, f"gradient {i}")


@pytest.mark.parametrize("dtype, M, K, N", [(BF16, 16_500, 72, 520), (F32, 16_500, 72, 520), (BF16, 4_200, 456, 2_056),
                                            (F16, 4_200, 640, 2_072), (F32, 4_200, 228, 2_060)])
def test_gated_large_tiles(dtype, M, K, N):
    g = gen(6)
    x, wg, wu = rand(g, M, K, dtype=dtype), rand(g, N, K, dtype=dtype, scale=0.1), rand(g, N, K, dtype=dtype, scale=0.1)
    grad = rand(g, M, N, dtype=dtype)
    want = ref.gated64(x, wg, wu, None, None, "gelu", None, grad)
    ref.check(geot.gated_linear(x, wg, wu, act="gelu"), *want[0], "out")
    for i, (t, w) in enumerate(zip(geot.gated_linear_backward(grad, x, wg, wu, act="gelu")[:3], want[1:])):
        ref.check(t, *w, f"gradient {i}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M, K, N, pad", [(17_000, 32, 256, 0), (20_001, 31, 300, 1), (16_385, 64, 20, 0), (9_000, 125, 130, 3),
                                          (9_001, 128, 40, 0), (8_200, 250, 260, 0), (8_300, 256, 9, 8), (30_000, 1, 70, 0),
                                          (3_000, 1032, 700, 0), (3_001, 1001, 705, 1), (100, 1032, 8_200, 0),
                                          (129, 1101, 4_100, 0), (9_001, 1101, 2_051, 0), (6_000, 1104, 1_024, 1)])
@pytest.mark.parametrize("act, bias, p", [("silu", True, 0.0), ("gelu", False, 0.25), ("relu", True, 0.5)])
def test_gated_many_rows(dtype, M, K, N, pad, act, bias, p):
    """Narrow rows (weights kept in registers, panels of columns, ragged tails of each) and wider ones, at odd and
    even addresses."""
    g = gen(M + K * 3 + N)
    x = rand(g, M, K, dtype=dtype, pad=pad)
    wg, wu = (rand(g, N, K, dtype=dtype, scale=1 / math.sqrt(K), pad=pad) for _ in range(2))
    bg, bu = (rand(g, N, dtype=dtype) if bias else None for _ in range(2))
    grad = rand(g, M, N, dtype=dtype, pad=pad)
    mask = mask_of(M, N, p) if p else None
    want = ref.gated64(x, wg, wu, bg, bu, act, mask, grad)
    ref.check(geot.gated_linear(x, wg, wu, bg, bu, act, p, SEED, OFFSET), *want[0], "out")
    for i, (t, w) in enumerate(zip(geot.gated_linear_backward(grad, x, wg, wu, bg, bu, act, p, SEED, OFFSET), want[1:])):
        if t is not None:
            ref.check(t, *w, f"gradient {i}")


@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("M, K, N, pad", [(700, 769, 693, 0), (1000, 1001, 900, 1), (300, 2051, 400, 3), (64, 770, 2731, 1),
                                          (30, 333, 700, 0), (5, 1003, 4100, 2), (1, 41, 9, 1)])
def test_gated_at_odd_addresses(dtype, M, K, N, pad):
    """Few rows or tiles over rows that start at any even address, alone and as a slice that starts at its second
    element, with NaN around it."""
    g = gen(M + K + N)
    wide = torch.full((M + 2 * N, K + pad + 1), math.nan, dtype=dtype, device=DEV)
    wide[:, 1:K + 1] = rand(g, M + 2 * N, K, dtype=dtype) / K ** 0.25
    x, wg, wu = (t[:, 1:K + 1] for t in (wide[:M], wide[M:M + N], wide[M + N:]))
    bg, bu, grad = rand(g, N, dtype=dtype), rand(g, N, dtype=dtype), rand(g, M, N, dtype=dtype)
    want = ref.gated64(x, wg, wu, bg, bu, "silu", None, grad)
    ref.check(geot.gated_linear(x, wg, wu, bg, bu), *want[0], "out")
    for i, (t, w) in enumerate(zip(geot.gated_linear_backward(grad, x, wg, wu, bg, bu), want[1:])):
        ref.check(t, *w, f"gradient {i}")
    cx, cg, cu = (t.contiguous() for t in (x, wg, wu))
    ref.check(geot.gated_linear(cx, cg, cu, bg, bu), *want[0], "out of whole tensors")


@pytest.mark.parametrize("M, K, N", [(700, 769, 693), (1000, 1001, 900), (1000, 1002, 900), (300, 2051, 400), (64, 770, 2731),
                                     (20, 333, 700), (5, 1003, 4100), (1, 41, 9)])
@pytest.mark.parametrize("at", [0, 1, 2, 3])
def test_int8_at_odd_addresses(M, K, N, at):
    g = gen(M * K + N)
    buf = torch.randint(-128, 128, ((M + N) * (K + 1) + at,), generator=g, device=DEV).to(torch.int8)
    both = buf[at:].view(M + N, K + 1)[:, :K]
    xq, wq = both[:M], both[M:]
    one_m, one_n = torch.ones(M, device=DEV), torch.ones(N, device=DEV)
    got = geot.linear_int8(xq, one_m, wq, one_n, dtype=F32)
    # sums below 2^24 in magnitude 2^14 K are not exact in fp32 beyond 1024 columns: half a last bit
    want = xq.double() @ wq.double().t()
    ref.check(got, want, torch.zeros_like(want), "out")


def test_gated_gradient_against_differences():
    """fp32 gradients against central differences of the block in 64 bits (whose error is of the order of h^2)."""
    M, K, N, h = 5, 9, 6, 1e-4
    g = gen(7)
    t = [rand(g, M, K), rand(g, N, K), rand(g, N, K), rand(g, N), rand(g, N)]
    grad, mask = rand(g, M, N), mask_of(M, N, 0.25)
    got = geot.gated_linear_backward(grad, *t, "silu", 0.25, SEED, OFFSET)
    wide = [v.double() for v in t]
    ref.EPS.setdefault(torch.float64, 2.0 ** -53)
    for i, (v, gv) in enumerate(zip(wide, got)):
        for j in range(v.numel()):
            at = []
            for s in (h, -h):
                moved = [w.clone() for w in wide]
                moved[i].view(-1)[j] += s
                at.append(float((ref.gated64(*moved, "silu", mask)[0][0] * grad).sum()))
            d = (at[0] - at[1]) / (2 * h)
            assert abs(d - float(gv.reshape(-1)[j])) <= 1e-4 * (1 + abs(d)), (i, j)


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_without_rows_or_columns(dtype):
    z = lambda *s: torch.zeros(s, dtype=dtype, device=DEV)  # noqa: E731
    one = torch.ones(4, dtype=dtype, device=DEV)
    assert geot.gated_linear(z(0, 8), z(4, 8), z(4, 8)).shape == (0, 4)
    assert geot.gated_linear(z(3, 8), z(0, 8), z(0, 8)).shape == (3, 0)
    out = geot.gated_linear(z(3, 0), z(4, 0), z(4, 0), one, one, act="relu")
    assert torch.equal(out, torch.ones_like(out))
    assert torch.equal(geot.gated_linear(z(3, 0), z(4, 0), z(4, 0)), z(3, 4))
    gx, gwg, gwu, gbg, gbu = geot.gated_linear_backward(z(0, 4), z(0, 8), z(4, 8), z(4, 8), one, one)
    assert gx.shape == (0, 8) and not gwg.any() and not gwu.any() and not gbg.any() and not gbu.any()
    gx, gwg, *_ = geot.gated_linear_backward(z(3, 0), z(3, 8), z(0, 8), z(0, 8))
    assert gx.shape == (3, 8) and not gx.any() and gwg.shape == (0, 8)
    gx, gwg, _, gbg, gbu = geot.gated_linear_backward(torch.ones(3, 4, dtype=dtype, device=DEV), z(3, 0), z(4, 0), z(4, 0), one,
                                                      one, act="none")
    assert gx.shape == (3, 0) and torch.equal(gbg, one * 3) and torch.equal(gbu, one * 3)


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_nan_stays_in_its_row(dtype):
    """A row with NaN or infinities spoils its own outputs alone, also where a tile or a part of K ends."""
    M, K, N = 70, 203, 37
    g = gen(8)
    x, wg, wu = rand(g, M, K, dtype=dtype), rand(g, N, K, dtype=dtype), rand(g, N, K, dtype=dtype)
    clean = geot.gated_linear(x, wg, wu)
    x2 = x.clone()
    x2[3, K - 1], x2[69, 0], x2[20, 100] = math.nan, math.inf, -math.inf
    got = geot.gated_linear(x2, wg, wu)
    rows = [i for i in range(M) if i not in (3, 20, 69)]
    assert torch.equal(got[rows], clean[rows]) and torch.isnan(got[3]).all()
    # beyond the rows and columns of a tensor that is a slice lies NaN, which nothing may read into a sum
    wide = torch.full((M + 3, K + 5), math.nan, device=DEV, dtype=dtype)
    wide[:M, :K] = x
    ww = torch.full((2 * N + 2, K + 5), math.nan, device=DEV, dtype=dtype)
    ww[:N, :K], ww[N + 1:2 * N + 1, :K] = wg, wu
    assert torch.equal(geot.gated_linear(wide[:M, :K], ww[:N, :K], ww[N + 1:2 * N + 1, :K]), clean)
    grad = rand(g, M, N, dtype=dtype)
    for a, b in zip(geot.gated_linear_backward(grad, wide[:M, :K], ww[:N, :K], ww[N + 1:2 * N + 1, :K]),
                    geot.gated_linear_backward(grad, x, wg, wu)):
        assert (a is None and b is None) or torch.equal(a, b)


def test_gated_writes_only_its_output():
    """Rows of a wider output keep what stands between them."""
    g = gen(9)
    x, w = rand(g, 37, 40, dtype=BF16), rand(g, 50, 40, dtype=BF16)
    wide = torch.full((40, 61), 7.0, device=DEV, dtype=BF16)
    geot.gated_linear(x, w[:25], w[25:], out=wide[1:38, 3:28])
    assert torch.equal(wide[1:38, 3:28], geot.gated_linear(x, w[:25], w[25:]))
    wide[1:38, 3:28] = 7.0
    assert (wide == 7).all()


def test_gated_far_strides():
    """Rows more than 2^32 bytes apart."""
    stride = (1 << 31) + 8
    base = torch.zeros(2 * stride + 64, dtype=BF16, device=DEV)
    x = torch.as_strided(base, (3, 64), (stride, 1))
    g = gen(10)
    x.copy_(rand(g, 3, 64, dtype=BF16))
    w = rand(g, 32, 64, dtype=BF16)
    assert torch.equal(geot.gated_linear(x, w[:16], w[16:]), geot.gated_linear(x.contiguous(), w[:16], w[16:]))
    del base, x
    torch.cuda.empty_cache()


def test_gated_is_reproducible():
    g = gen(11)
    x, w, grad = rand(g, 5000, 96), rand(g, 80, 96), rand(g, 5000, 40)
    a = geot.gated_linear_backward(grad, x, w[:40], w[40:], w[:40, 0].contiguous(), None)
    for _ in range(3):
        b = geot.gated_linear_backward(grad, x, w[:40], w[40:], w[:40, 0].contiguous(), None)
        assert all(torch.equal(p, q) for p, q in zip(a[:4], b[:4]))


# ---- 8 bits ----------------------------------------------------------------
def quantize_np(x):
    x = x.float().cpu().numpy()
    a = np.maximum(np.abs(x).max(axis=1, initial=0.0), np.float32(2.0 ** -100)).astype(np.float32)
    k = (np.float32(127.0) / a).astype(np.float32)
    return np.rint(x * k[:, None]).astype(np.int8), (a / np.float32(127.0)).astype(np.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, F, pad", [(1, 1, 0), (1, 4096, 0), (3, 7, 0), (5, 1001, 3), (130, 64, 0), (2, 9000, 0), (4000, 12, 1),
                                          (2, 40_001, 0), (3, 0, 0)])
def test_quantize(dtype, rows, F, pad):
    x = rand(gen(F + rows), rows, F, dtype=dtype, pad=pad)
    x[0] *= 100
    if rows > 2:
        x[1], x[2] = 0, x[2] * 1e-5
    q, scale = geot.quantize_rows(x)
    wq, ws = quantize_np(x)
    assert np.array_equal(scale.cpu().numpy(), ws) and np.array_equal(q.cpu().numpy(), wq)
    if F:
        assert ((q.double() * scale.double()[:, None] - x.double()).abs() <= scale.double()[:, None] * (0.5 + 1e-4)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_rows_without_a_scale(dtype):
    x = torch.ones(6, 20, dtype=dtype, device=DEV)
    x[1, 19], x[3, 0], x[4, 7] = math.nan, math.inf, -math.inf
    q, scale = geot.quantize_rows(x)
    assert torch.isnan(scale[[1, 3, 4]]).all() and not q[[1, 3, 4]].any()
    assert (q[[0, 2, 5]] == 127).all() and torch.isfinite(scale[[0, 2, 5]]).all()
    w, sw = geot.quantize_rows(torch.ones(5, 20, device=DEV))
    out = geot.linear_int8(q, scale, w, sw, dtype=F32)
    assert torch.isnan(out[[1, 3, 4]]).all() and torch.isfinite(out[[0, 2, 5]]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M, K, N, pad, bias", [(1, 1, 1, 0, False), (1, 4096, 520, 0, True), (2, 15, 3, 1, True), (7, 1001, 66, 0, True),
                                               (17, 128, 16, 16, False), (33, 130, 200, 5, True), (333, 1500, 130, 0, True),
                                               (300, 48, 1000, 0, False), (129, 257, 129, 0, True), (1, 131071, 5, 0, False),
                                               (8, 2064, 96, 0, True), (16, 96, 3000, 0, False)])
def test_int8(dtype, M, K, N, pad, bias):
    g = gen(M + K * 7 + N)
    xq = torch.randint(-128, 128, (M, K + pad), generator=g, device=DEV).to(torch.int8)[:, :K]
    wq = torch.randint(-128, 128, (N, K + pad), generator=g, device=DEV).to(torch.int8)[:, :K]
    sx, sw = torch.rand(M, generator=g, device=DEV) * 1e-2, torch.rand(N, generator=g, device=DEV) * 1e-2
    b = torch.randn(N, generator=g, device=DEV) if bias else None
    got = geot.linear_int8(xq, sx, wq, sw, b, dtype=dtype)
    y = (xq.double() @ wq.double().t()) * sx.double()[:, None] * sw.double()
    want = y + b.double() if bias else y
    ref.check(got, want, 4 * ref.U * (y.abs() + want.abs()), "int8")


def test_int8_extreme_sums():
    """The longest sums of the largest products stay exact."""
    K = 131071
    xq, wq = (torch.full((2, K), -128, dtype=torch.int8, device=DEV) for _ in range(2))
    one = torch.ones(2, device=DEV)
    got = geot.linear_int8(xq, one, wq, one, dtype=F32)
    assert (got.double() == float(np.float32(128.0 * 128.0 * K))).all()


@pytest.mark.parametrize("M, K, N", [(5000, 200, 4100), (5000, 1040, 4100), (5000, 1280, 4100), (100, 4112, 16_400), (1500, 2001, 1700),
                                     (3001, 2117, 3203)])
def test_int8_large_tiles(M, K, N):
    g = gen(12)
    xq = torch.randint(-127, 128, (M, K), generator=g, device=DEV).to(torch.int8)
    wq = torch.randint(-127, 128, (N, K), generator=g, device=DEV).to(torch.int8)
    sx, sw = torch.rand(M, generator=g, device=DEV), torch.rand(N, generator=g, device=DEV)
    y = (xq.double() @ wq.double().t()) * sx.double()[:, None] * sw.double()
    ref.check(geot.linear_int8(xq, sx, wq, sw, dtype=F32), y, 4 * ref.U * y.abs(), "int8")


# ---- as a program runs them ------------------------------------------------
def test_on_other_streams_and_in_graphs():
    """Calls on a side stream, and a captured step replayed between eager work, give the eager results."""
    g = gen(13)
    x, w, b, grad = rand(g, 600, 72, dtype=BF16), rand(g, 256, 72, dtype=BF16), rand(g, 128, dtype=BF16), rand(g, 600, 128, dtype=BF16)
    wq, sw = geot.quantize_rows(w)

    def step():
        y = geot.gated_linear(x, w[:128], w[128:], b, b, "silu", 0.25, SEED, 4)
        grads = geot.gated_linear_backward(grad, x, w[:128], w[128:], b, b, "silu", 0.25, SEED, 4)
        d = geot.dropout(y, 0.5, SEED, 5, residual=y)
        return [y, d, *grads, geot.linear_int8(*geot.quantize_rows(x), wq, sw), geot.gated_linear(x[:1], w[:128], w[128:])]

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        kept = step()
    for i in range(4):
        for t in kept:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(kept, want)), i
        again = step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(again, want)), i


def graph_of(g, nodes=300, edges=2000):
    row = torch.randint(0, nodes, (edges,), generator=g, device=DEV).sort().values
    col = torch.randint(0, nodes, (edges,), generator=g, device=DEV)
    return ga.Graph(col, row, nodes)


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_gated_conv(dtype):
    """The layer against the same layer from plain operations in 64 bits, forward and every gradient."""
    g = gen(14)
    graph, D, H, p = graph_of(g), 40, 72, 0.25
    torch.manual_seed(1)
    layer = ga.GatedConv(D, H, p=p, seed=77).to(DEV).to(dtype)
    h = rand(g, 300, D, dtype=dtype).requires_grad_(True)
    up = rand(g, 300, D, dtype=dtype)
    layer.train()
    out = layer(h, graph)
    out.backward(up)
    m1, m2 = mask_of(300, H, p, 77, 0), mask_of(300, D, p, 77, 1)
    ps = {k: v.detach().double().requires_grad_(True) for k, v in layer.named_parameters()}
    hd = h.detach().double().requires_grad_(True)
    count = torch.bincount(graph.row, minlength=300).clamp_min(1)
    z = torch.zeros(300, D, dtype=torch.float64, device=DEV).index_add(0, graph.row, hd[graph.col]) / count[:, None]
    y = torch.nn.functional.silu(z @ ps["gate.weight"].t() + ps["gate.bias"]) * (z @ ps["up.weight"].t() + ps["up.bias"]) * m1
    want = hd + m2 * (y @ ps["down.weight"].t())
    want.backward(up.double())
    # chains of five rounded steps: 16 units of the type's last bit, relative to the tensor's size
    lim = 16 * 2 * ref.EPS[dtype]
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert rel(out, want) <= lim and rel(h.grad, hd.grad) <= lim
    for k, v in layer.named_parameters():
        assert rel(v.grad, ps[k].grad) <= lim, k
    # the next call drops others; evaluation drops none, and 8 bits stay near it
    assert not torch.equal(layer(h, graph), out)
    layer.eval()
    with torch.no_grad():
        plain, small = layer(h, graph), layer.int8()(h, graph)
    # two operands rounded to 1/254 of their largest: the difference from the residual is a few percent
    assert rel(small - h.detach(), (plain - h.detach()).double()) <= 0.05


def test_gated_conv_learns():
    """A few steps of a small classifier with two layers lower its loss."""
    g = gen(15)
    graph = graph_of(g)
    torch.manual_seed(2)
    net = torch.nn.ModuleList([ga.GatedConv(32, 64, p=0.1), ga.GatedConv(32, 64, p=0.1)]).to(DEV)
    head = torch.nn.Linear(32, 5).to(DEV)
    x, y = rand(g, 300, 32), torch.randint(0, 5, (300,), generator=g, device=DEV)
    opt = torch.optim.Adam([*net.parameters(), *head.parameters()], lr=1e-2)
    losses = []
    for _ in range(30):
        h = x
        for layer in net:
            h = layer(h, graph)
        loss = torch.nn.functional.cross_entropy(head(h), y)
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    assert losses[-1] < 0.7 * losses[0], losses
