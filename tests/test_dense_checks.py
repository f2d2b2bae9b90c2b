"""The dense operators' argument checks and their generator, on the CPU: shapes and types in the binding, sizes,
strides, alignment and overlaps at the C entry points (pointers there are never dereferenced)."""
import numpy as np
import pytest
import torch

import paper_2404_03019_amd as geot
from paper_2404_03019_amd import autograd as ga
from paper_2404_03019_amd.geot import lib

import dense_ref as ref

SUCCESS, INVALID = 0, 1
FAR = 1 << 36


def ptr(i):
    return 0x10000000 + i * FAR


def detail():
    return lib().geot_last_error_detail().decode()


def drop(x=ptr(0), type=0, rows=4, F=8, ldx=8, res=None, ldr=8, p=0.5, out=ptr(1), ldo=8):
    return lib().geot_dropout(x, type, rows, F, ldx, res, ldr, p, 1, 2, out, ldo, None)


def gated(x=ptr(0), type=1, M=4, K=8, ldx=8, wg=ptr(1), wu=ptr(2), N=6, ldw=8, bg=None, bu=None, act=0, p=0.0,
          out=ptr(3), ldo=6):
    return lib().geot_gated_linear(x, type, M, K, ldx, wg, wu, N, ldw, bg, bu, act, p, 1, 2, out, ldo, None)


def gated_back(grad=ptr(3), ldg=6, x=ptr(0), type=1, M=4, K=8, ldx=8, wg=ptr(1), wu=ptr(2), N=6, ldw=8, act=0, p=0.0,
               gx=ptr(4), gwg=ptr(5), gwu=ptr(6), gbg=None, gbu=None):
    return lib().geot_gated_linear_backward(grad, ldg, x, type, M, K, ldx, wg, wu, N, ldw, None, None, act, p, 1, 2, gx,
                                            gwg, gwu, gbg, gbu, None)


def quant(x=ptr(0), type=1, rows=4, F=8, ldx=8, q=ptr(1), ldq=8, scale=ptr(2)):
    return lib().geot_quantize_rows(x, type, rows, F, ldx, q, ldq, scale, None)


def int8(xq=ptr(0), sx=ptr(1), M=4, K=8, ldx=8, wq=ptr(2), sw=ptr(3), N=6, ldw=8, bias=None, out=ptr(4), type=1, ldo=6):
    return lib().geot_linear_int8(xq, sx, M, K, ldx, wq, sw, N, ldw, bias, out, type, ldo, None)


@pytest.mark.parametrize("call, args, word", [
    (drop, dict(type=3), "type"), (drop, dict(rows=-1), "negative"), (drop, dict(F=-1), "negative"),
    (drop, dict(x=None), "x is NULL"), (drop, dict(out=None), "out is NULL"), (drop, dict(ldx=7), "row stride"),
    (drop, dict(ldo=7), "row stride"), (drop, dict(res=ptr(2), ldr=7), "row stride"), (drop, dict(x=ptr(0) + 2), "aligned"),
    (drop, dict(p=-0.1), "p must"), (drop, dict(p=1.1), "p must"), (drop, dict(p=float("nan")), "p must"),
    (drop, dict(out=ptr(0) + 16), "overlaps x"), (drop, dict(out=ptr(0), ldo=9), "overlaps x"),
    (drop, dict(res=ptr(1) + 16), "overlaps residual"), (drop, dict(rows=1 << 60), "overflow"),
    (drop, dict(rows=(1 << 32) + 1, F=1, ldx=1, ldo=1), "2^32 rows"),
    (gated, dict(type=7), "type"), (gated, dict(act=5), "activation"), (gated, dict(act=-1), "activation"),
    (gated, dict(M=-1), "negative"), (gated, dict(K=-1), "negative"), (gated, dict(N=-1), "negative"),
    (gated, dict(x=None), "x is NULL"), (gated, dict(wg=None), "w_gate is NULL"), (gated, dict(wu=None), "w_up is NULL"),
    (gated, dict(out=None), "out is NULL"), (gated, dict(ldx=7), "row stride"), (gated, dict(ldw=7), "row stride"),
    (gated, dict(ldo=5), "row stride"), (gated, dict(p=2.0), "p must"), (gated, dict(out=ptr(0)), "overlaps x"),
    (gated, dict(out=ptr(1) + 8), "overlaps w_gate"), (gated, dict(out=ptr(2)), "overlaps w_up"),
    (gated, dict(bg=ptr(3) + 4), "overlaps b_gate"), (gated, dict(bu=ptr(3)), "overlaps b_up"),
    (gated, dict(bg=ptr(7) + 1), "bias is not aligned"), (gated, dict(wg=ptr(1) + 1), "aligned"),
    (gated_back, dict(grad=None), "grad_out is NULL"), (gated_back, dict(ldg=5), "row stride"),
    (gated_back, dict(gwu=None), "go together"), (gated_back, dict(gwg=None), "go together"),
    (gated_back, dict(gx=ptr(0)), "overlaps x"), (gated_back, dict(gx=ptr(3)), "overlaps grad_out"),
    (gated_back, dict(gwu=ptr(5) + 32), "overlaps grad_w_gate"), (gated_back, dict(gbg=ptr(4)), "overlaps grad_x"),
    (gated_back, dict(p=1.5), "p must"), (gated_back, dict(act=9), "activation"),
    (quant, dict(type=-1), "type"), (quant, dict(x=None), "x is NULL"), (quant, dict(q=None), "q is NULL"),
    (quant, dict(scale=None), "scale is NULL"), (quant, dict(ldx=7), "row stride"), (quant, dict(ldq=7), "row stride"),
    (quant, dict(q=ptr(0)), "overlaps x"), (quant, dict(scale=ptr(1)), "overlaps q"), (quant, dict(scale=ptr(2) + 2), "aligned"),
    (int8, dict(type=4), "type"), (int8, dict(xq=None), "xq is NULL"), (int8, dict(wq=None), "wq is NULL"),
    (int8, dict(sx=None), "x_scale is NULL"), (int8, dict(sw=None), "w_scale is NULL"), (int8, dict(out=None), "out is NULL"),
    (int8, dict(ldx=7), "row stride"), (int8, dict(ldw=7), "row stride"), (int8, dict(ldo=5), "row stride"),
    (int8, dict(K=131072, ldx=131072, ldw=131072), "131071"), (int8, dict(out=ptr(2)), "overlaps wq"),
    (int8, dict(bias=ptr(4)), "overlaps bias"), (int8, dict(bias=ptr(5) + 1), "aligned"),
])
def test_refused_on_the_host(call, args, word):
    assert call(**args) == INVALID
    assert word in detail(), detail()


@pytest.mark.parametrize("call, args", [
    (drop, dict(rows=0, x=None, out=None)), (drop, dict(F=0, x=None, out=None)), (gated, dict(M=0, x=None, out=None)),
    (gated, dict(N=0, wg=None, wu=None, out=None)), (gated_back, dict(gx=None, gwg=None, gwu=None)),
    (quant, dict(rows=0, x=None, q=None, scale=None)), (int8, dict(M=0, xq=None, sx=None, out=None)),
    (int8, dict(N=0, wq=None, sw=None, out=None)),
])
def test_nothing_to_do(call, args):
    assert call(**args) == SUCCESS


def test_binding_shapes():
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    with pytest.raises(ValueError, match="residual must have shape"):
        geot.dropout(f(3, 4), 0.5, 1, residual=f(3, 5))
    with pytest.raises(TypeError, match="residual"):
        geot.dropout(f(3, 4), 0.5, 1, residual=f(3, 4, dtype=torch.float16))
    with pytest.raises(ValueError, match="unit stride"):
        geot.dropout(f(4, 3).t(), 0.5, 1)
    with pytest.raises(ValueError, match="do not overlap"):
        geot.dropout(f(1, 4).expand(3, 4), 0.5, 1)
    with pytest.raises(ValueError, match="p must"):
        geot.dropout(f(3, 4), 1.5, 1)
    with pytest.raises(TypeError):
        geot.dropout(f(3, 4, dtype=torch.float64), 0.5, 1)
    with pytest.raises(ValueError, match="dimensions"):
        geot.dropout(f(2, 3, 4), 0.5, 1)
    for bad in (dict(x=f(3, 5)), dict(w_up=f(6, 5)), dict(w_up=f(7, 4)), dict(b_gate=f(5)), dict(b_up=f(6, 1)),
                dict(act="tanh"), dict(p=-1.0), dict(out=f(3, 7)), dict(w_up=f(6, 8)[:, :4]), dict(x=f(4))):
        with pytest.raises(ValueError):
            geot.gated_linear(**(dict(x=f(3, 4), w_gate=f(6, 4), w_up=f(6, 4)) | bad))
    with pytest.raises(TypeError):
        geot.gated_linear(f(3, 4), f(6, 4, dtype=torch.bfloat16), f(6, 4))
    with pytest.raises(ValueError, match="grad_out must have shape"):
        geot.gated_linear_backward(f(3, 5), f(3, 4), f(6, 4), f(6, 4))
    b = lambda *s: torch.zeros(s, dtype=torch.int8)  # noqa: E731
    for bad in (dict(xq=b(3, 5)), dict(x_scale=f(4)), dict(w_scale=f(5)), dict(bias=f(5)), dict(out=f(3, 5))):
        with pytest.raises(ValueError):
            geot.linear_int8(**(dict(xq=b(3, 4), x_scale=f(3), wq=b(6, 4), w_scale=f(6), dtype=torch.float32) | bad))
    for bad in (dict(xq=f(3, 4)), dict(dtype=torch.int32), dict(w_scale=f(6, dtype=torch.float16))):
        with pytest.raises(TypeError):
            geot.linear_int8(**(dict(xq=b(3, 4), x_scale=f(3), wq=b(6, 4), w_scale=f(6)) | bad))
    for call in (lambda: geot.dropout(f(3, 4), 0.5, 1), lambda: geot.gated_linear(f(3, 4), f(6, 4), f(6, 4)),
                 lambda: geot.quantize_rows(f(3, 4)), lambda: geot.linear_int8(b(3, 4), f(3), b(6, 4), f(6)),
                 lambda: ga.GatedConv(4, 6)(f(3, 4), torch.zeros(5, dtype=torch.int64), torch.zeros(5, dtype=torch.int64), 3)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
    with pytest.raises(ValueError, match="same nodes"):
        ga.GatedConv(4, 6)(f(3, 4), torch.zeros(5, dtype=torch.int64), torch.zeros(5, dtype=torch.int64), 2)


def test_reference_generator():
    """The oracle's generator gives the published vectors of Philox4x32 (7 and 10 rounds)."""
    zero = np.zeros((1, 4), dtype=np.uint64)
    assert [int(v) for v in ref.philox(zero, (0, 0), 7)[0]] == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    assert [int(v) for v in ref.philox(zero, (0, 0), 10)[0]] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    m = 0xFFFFFFFF
    ones = np.full((1, 4), m, dtype=np.uint64)
    assert [int(v) for v in ref.philox(ones, (m, m), 10)[0]] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_reference_gradients_against_differences():
    """The formulas of the gradients against central differences of the block, in 64 bits."""
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)  # noqa: E731
    M, K, N, h = 3, 5, 4, 1e-5
    for act in ("silu", "gelu", "relu", "sigmoid", "none"):
        t = [r(M, K), r(N, K), r(N, K), r(N), r(N)]
        mask = (torch.rand(M, N, generator=gen) < 0.7).double() / 0.7
        grad = r(M, N)
        ref.EPS.setdefault(torch.float64, 2.0 ** -53)
        ref.TINY.setdefault(torch.float64, 0.0)
        want = [v for v, _ in ref.gated64(*t, act, mask, grad)][1:]
        for i, (v, g) in enumerate(zip(t, want)):
            for j in range(v.numel()):
                at = []
                for s in (h, -h):
                    moved = [w.clone() for w in t]
                    moved[i].view(-1)[j] += s
                    at.append(float((ref.gated64(*moved, act, mask)[0][0] * grad).sum()))
                d = (at[0] - at[1]) / (2 * h)
                # h^2 of the third derivative, and the differences' own rounding
                assert abs(d - float(g.reshape(-1)[j])) <= 1e-6 * (1 + abs(d)), (act, i, j)
