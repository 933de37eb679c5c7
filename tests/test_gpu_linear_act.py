"""The bf16 product with bias, activation and residual, on the GPU.

Against 64 bits. Tolerance: the output's rounding 2^-8 |ref|, and before it the
fp32 steps: the sum of K exact products in any order, K u sum|a w| (u = 2^-24); x =
sum + bias (u relative to |x|, which with the sum's error an activation of slope at
most 1.13 passes on), the activation's hardware exp2 and reciprocal with the
rounding of its argument (|x| u + 8 u relative for SiLU's and tanh-GELU's
exponential, whose cube adds 3 u |argument|), erf's formula (0.75e-7 |x|), SwiGLU's product
and the residual's addition (u each)."""

import math

import pytest
import torch

import paper_2607_16339_amd as lc
from paged_util import DEV, normal

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NONE, RELU, SILU, GELU, GELU_TANH, SWIGLU = range(6)


def _act(act, x, off):
    """(value, its tolerance) of the activation of x, which is off by u |x| and `off`."""
    slack = 1.2 * (U * x.abs() + off)
    if act == RELU:
        return x.clamp_min(0.0), slack
    if act in (SILU, SWIGLU):
        y = x * torch.sigmoid(x)
        return y, slack + y.abs() * (3 * x.abs() + 8) * U
    if act == GELU:
        return 0.5 * x * torch.erfc(-x / math.sqrt(2.0)), slack + x.abs() * (0.75e-7 + 8 * U)
    if act == GELU_TANH:
        w = 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
        y = x * torch.sigmoid(w)
        return y, slack + y.abs() * (5 * w.abs() + 8) * U
    return x, slack


def _case(M, N, K, act, bias, residual, seed=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    rows = 2 * N if act == SWIGLU else N
    a, w = normal(g, (M, K), std).to(DEV), normal(g, (rows, K), 0.05).to(DEV)
    b = normal(g, (rows,), 0.5).to(DEV) if bias else None
    r = normal(g, (M, N), 2.0).to(DEV) if residual else None
    return a, w, b, r


def _want(a, w, b, r, act):
    rows = w.shape[0]
    wt = w.double().t().contiguous()
    x = a.double() @ wt
    off = a.shape[1] * U * (a.double().abs() @ wt.abs())
    if b is not None:
        x = x + b.double()
    if act == SWIGLU:
        N = rows // 2
        y, t = _act(SWIGLU, x[:, :N], off[:, :N])
        u, du = x[:, N:], off[:, N:]
        t = t * (u.abs() + du) + y.abs() * (u.abs() * 3 * U + du)
        y = y * u
    else:
        y, t = _act(act, x, off)
    if r is not None:
        y = y + r.double()
        t = t + U * y.abs()
    return y, t * (1 + 2.0 ** -7) + 2.0 ** -8 * y.abs() + 1e-38


def _check(M, N, K, act, bias, residual, seed=0, std=1.0, in_place=False):
    a, w, b, r = _case(M, N, K, act, bias, residual, seed, std)
    want, tol = _want(a, w, b, r, act)
    buf = torch.full((M * N + 256,), 7.0, dtype=torch.bfloat16, device=DEV)
    out = buf[128:128 + M * N].view(M, N)
    if in_place:
        out.copy_(r)
        lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=out, act=act)
    else:
        lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=r, act=act)
    torch.cuda.synchronize()
    assert bool((buf[:128] == 7).all()) and bool((buf[128 + M * N:] == 7).all())
    err = (out.double() - want).abs()
    worst = float((err / tol).max())
    print("M %d N %d K %d act %d: worst err/tolerance %.3f" % (M, N, K, act, worst), flush=True)
    assert worst <= 1.0
    return out


# 1 to 4 slabs streamed, two passes, and tiles, with ragged ends
ROWS = [1, 2, 16, 17, 32, 33, 48, 64, 65, 100, 128, 129, 200, 257, 1000]


@pytest.mark.parametrize("act", range(6))
@pytest.mark.parametrize("M", ROWS)
def test_rows_and_activations(M, act):
    _check(M, 384, 256, act, True, True, seed=M)


@pytest.mark.parametrize("act", [GELU, SWIGLU])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("M", [5, 70, 300])
def test_optional_operands(M, bias, residual, act):
    _check(M, 256, 128, act, bias, residual, seed=M + 1)


@pytest.mark.parametrize("act", [NONE, SILU, SWIGLU])
@pytest.mark.parametrize("M,N,K", [(1, 128, 128), (8, 12288, 256), (32, 12288, 512), (20, 128, 8192), (130, 128, 128),
                                   (700, 1152, 640), (1500, 12288, 128), (2100, 3840, 192 * 2), (300, 640, 1024)])
def test_sizes(M, N, K, act):
    _check(M, N, K, act, True, True, seed=N + K)


@pytest.mark.parametrize("M", [3, 40, 128, 129, 600])
@pytest.mark.parametrize("act", [NONE, GELU_TANH, SWIGLU])
def test_residual_updated_in_place(M, act):
    x = _check(M, 256, 256, act, True, True, seed=M, in_place=True)
    y = _check(M, 256, 256, act, True, True, seed=M)
    assert torch.equal(x.view(torch.int16), y.view(torch.int16))


# (M, N, K) of each tile and of the streaming kernel; ragged rows, and columns where the tile is wider than what is left
TILES = {(64, 16): [(7, 1024, 4096), (100, 1024, 4096)], (64, 48): [(20, 12288, 4096)],
         (32, 64): [(60, 1152, 640), (96, 4096, 2048)], (64, 64): [(90, 6144, 2048), (50, 12288, 512)],
         (64, 128): [(300, 4224, 512), (1500, 1024, 1024)], (128, 128): [(1000, 4096, 256), (1300, 2944, 512)],
         (128, 256): [(2047, 4096, 384), (2040, 3968, 1024), (2040, 3968, 2048), (777, 8064, 2048)], (256, 256): [(8000, 4096, 1024), (6000, 2176, 2048)]}


@pytest.mark.parametrize("tile", sorted(TILES))
@pytest.mark.parametrize("act", [NONE, GELU, SWIGLU])
def test_tiles(tile, act):
    for M, N, K in TILES[tile]:
        if act == SWIGLU:
            N = max(128, N // 2 // 128 * 128)
        assert act == SWIGLU or lc.lacache_linear_act_tile(M, N, K, act) == tile
        _check(M, N, K, act, True, True, seed=M + N)


@pytest.mark.parametrize("act", [NONE, SWIGLU])
def test_rows_do_not_depend_on_the_call(act):
    """The first rows of calls of more than 128 rows, on every tile, are the same bytes."""
    a, w, b, r = _case(8192, 1024, 1024, act, True, True, seed=3)
    seen, first = set(), None
    for M in (129, 200, 700, 1500, 3000, 8192):
        out = torch.empty((M, 1024), dtype=torch.bfloat16, device=DEV)
        lc.lacache_linear_act_bf16(a[:M], w, out, bias=b, residual=r[:M], act=act)
        seen.add(lc.lacache_linear_act_tile(M, 1024, 1024, act))
        first = out[:129].clone() if first is None else first
        assert torch.equal(out[:129].view(torch.int16), first.view(torch.int16)), M
    print(sorted(seen))
    assert len(seen) >= 4


@pytest.mark.parametrize("act", [NONE, SWIGLU])
def test_rows_do_not_depend_on_the_call_at_a_longer_k(act):
    a, w, b, r = _case(8192, 1024, 4096, act, True, True, seed=5)
    seen, first = set(), None
    for M in (129, 700, 1500, 3000, 4096, 8192):
        out = torch.empty((M, 1024), dtype=torch.bfloat16, device=DEV)
        lc.lacache_linear_act_bf16(a[:M], w, out, bias=b, residual=r[:M], act=act)
        seen.add(lc.lacache_linear_act_tile(M, 1024, 4096, act))
        first = out[:129].clone() if first is None else first
        assert torch.equal(out[:129].view(torch.int16), first.view(torch.int16)), M
    assert (128, 256) in seen and len(seen) >= 3


@pytest.mark.parametrize("M", [1, 16, 33, 64, 100, 128])
def test_streamed_product_is_the_plain_one_bit_for_bit(M):
    assert lc.lacache_linear_act_tile(M, 1024, 4096)[1] in (16, 48)
    a, w, _, _ = _case(M, 1024, 4096, NONE, False, False, seed=M)
    a[0, 3] = float("nan")
    out, plain = (torch.empty((M, 1024), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lc.lacache_linear_act_bf16(a, w, out)
    lc.lacache_linear_bf16(a, w, plain)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), plain.view(torch.int16))


@pytest.mark.parametrize("act", range(6))
@pytest.mark.parametrize("M", [4, 200])
def test_far_arguments_and_values_that_are_no_numbers(M, act):
    """Sums of hundreds, where exp overflows; infinities and NaNs pass like the formula's."""
    _check(M, 256, 256, act, True, False, seed=9, std=300.0)
    a, w, b, r = _case(M, 128, 128, act, True, True, seed=10)
    b[0], b[1], b[2] = float("inf"), float("-inf"), float("nan")
    out = torch.empty((M, 128), dtype=torch.bfloat16, device=DEV)
    lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=r, act=act)
    torch.cuda.synchronize()
    o = out.float()
    assert bool((o[:, 0].abs() == math.inf).all()) and bool(torch.isfinite(o[:, 3:]).all())
    assert bool(torch.isnan(o[:, 2]).all()) and bool((out[:, 2].view(torch.int16) == 0x7FC0).all())
    if act == NONE:
        assert bool((o[:, 1] == -math.inf).all())


def test_captured_and_replayed():
    a, w, b, r = _case(40, 256, 256, SILU, True, True, seed=11)
    out = torch.empty((40, 256), dtype=torch.bfloat16, device=DEV)
    lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=r, act=SILU)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=r, act=SILU)
    for k in range(3):
        a.mul_(-0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=r, act=SILU)
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), out.view(torch.int16)), k
