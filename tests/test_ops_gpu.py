"""The operators of include/gecc_ops.h against their plain 64-bit forms (tests/ops_reference.py).

Tolerances.  Quantised matrices: byte for byte.  Products: the terms are exact, their sums are fp32; |C - C64| <= 2^-23 k
max over the element's own sum of |terms| (k additions, each within half an ulp of a running sum no larger than that; the
factor of two for sums that a matrix instruction forms its own way), plus half an ulp of bfloat16 (8 significant bits: 2^-8) where the output is.
Sums whose terms fit 24 bits together have to be exact.  Orthogonalised updates, in the Frobenius norm: a step rounds X, S and
its polynomial to 11 bits (2^-12 of the value each, rms), five steps make 15 such roundings, and the polynomial's slope on what
is near its fixed points is below 1.4 in the mean: 15 * 2^-12 * 1.4 = 5.1e-3; bfloat16 outputs 2^-9 more (rms)."""
import numpy as np
import pytest
import torch

import ops_reference as R
from paper_2508_04355_amd import gecc, ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
ORTH_TOL, ORTH_BF16, BF16_TOL = 5.2e-3, 2.0 ** -9, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rng(*key):
    return np.random.default_rng([7, *key])


def _store(x, dtype):
    """x as the type stores it (numpy float32) and on the GPU."""
    x = R.bf16(x) if dtype == "bf16" else np.asarray(x, np.float32)
    return x, torch.from_numpy(x).to(DEV).to(DT[dtype])


def _values_of(q):
    return ops.mx4_dequantize(q, torch.float32).double().cpu().numpy()


def _matrix(rng, rows, cols, kind="normal"):
    x = rng.standard_normal((rows, cols))
    if kind == "wide":          # magnitudes over the whole range of the type, zeros and signs of zero among them
        x = np.ldexp(x, rng.integers(-140, 120, (rows, cols)))
        x[rng.random((rows, cols)) < 0.1] = 0.0
        x[rng.random((rows, cols)) < 0.05] = -0.0
    elif kind == "ties":
        x = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0, 6.5, 7.75], (rows, cols)) * rng.choice([-1.0, 1.0], (rows, cols))
    return x


# ---- quantisation ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "wide", "ties"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (1, 33), (3, 256), (16, 512), (17, 513), (33, 100), (129, 65), (200, 776), (257, 1025), (1, 4096), (1000, 7)])
def test_quantised_bytes(rows, cols, kind, dtype):
    x, t = _store(_matrix(_rng(rows, cols), rows, cols, kind), dtype)
    data, scales = R.packed(*R.quantise(x))
    tdata, tscales = R.packed(*R.quantise(x.T))
    q, qt = ops.mx4_quantize(t, both=True)
    alone = ops.mx4_quantize(t)
    for got, want in ((q.data, data), (q.scales, scales), (qt.data, tdata), (qt.scales, tscales), (alone.data, data), (alone.scales, scales)):
        assert np.array_equal(got.cpu().numpy().ravel(), want.ravel())
    want = R.values(*R.quantise(x))
    assert np.array_equal(_values_of(q), want)
    assert np.array_equal(ops.mx4_dequantize(q).double().cpu().numpy(), want)


def test_only_the_transpose_through_the_c_abi():
    x, t = _store(_matrix(_rng(1), 70, 300), "f32")
    want = ops.mx4_quantize(t, both=True)[1]
    got = ops.Mx4._new(300, 70, t.device)
    gecc._check(ops.lib().gecc_mx4_quantize(t.data_ptr(), 0, 70, 300, 300, 0, 0, got.data.data_ptr(), got.scales.data_ptr(), gecc._stream()))
    assert torch.equal(got.data, want.data) and torch.equal(got.scales, want.scales)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_start_anywhere(dtype):
    """Views with odd leading dimensions and odd first elements: nothing beyond the view's columns is read."""
    big = torch.full((40, 1003), float("nan"), device=DEV, dtype=DT[dtype])
    x, t = _store(_matrix(_rng(2), 37, 500), dtype)
    view = big[2:39, 301:801]
    view.copy_(t)
    a, at = ops.mx4_quantize(view, both=True)
    b, bt = ops.mx4_quantize(t, both=True)
    for u, v in ((a, b), (at, bt)):
        assert torch.equal(u.data, v.data) and torch.equal(u.scales, v.scales)
    out = torch.full((40, 1003), 7.0, device=DEV, dtype=DT[dtype])
    ops.mx4_dequantize(a, out=out[2:39, 301:801])
    assert torch.equal(out[2:39, 301:801], ops.mx4_dequantize(b, DT[dtype]))
    out[2:39, 301:801] = 7.0
    assert bool((out == 7.0).all())
    c = ops.mx4_quantize(t.t().contiguous().t())           # columns contiguous: a copy is quantised
    assert torch.equal(c.data, b.data)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_blocks_that_hold_no_number(dtype, value):
    x, t = _store(_matrix(_rng(3), 40, 200), dtype)
    x[5, 70] = value
    t[5, 70] = value
    q, qt = ops.mx4_quantize(t, both=True)
    want = R.rounded(x)
    assert np.isnan(want[5, 64:96]).all() and np.isnan(want).sum() == 32
    assert np.array_equal(_values_of(q), want, equal_nan=True)
    assert np.array_equal(_values_of(qt), R.rounded(x.T), equal_nan=True)
    y = ops.mx4_gemm(q, ops.mx4_quantize(_store(_matrix(_rng(4), 70, 200), dtype)[1])).cpu().numpy()
    assert np.isnan(y[5]).all() and np.isfinite(np.delete(y, 5, axis=0)).all()


def test_offsets_beyond_32_bits():
    ld = (1 << 30) + 8
    big = torch.empty(2 * ld + 600, dtype=torch.bfloat16, device=DEV)
    view = big.as_strided((3, 600), (ld, 1))
    x, t = _store(_matrix(_rng(5), 3, 600), "bf16")
    view.copy_(t)
    a, at = ops.mx4_quantize(view, both=True)
    b, bt = ops.mx4_quantize(t, both=True)
    assert torch.equal(a.data, b.data) and torch.equal(at.data, bt.data) and torch.equal(a.scales, b.scales)
    ops.mx4_dequantize(b, out=view)
    assert torch.equal(view, ops.mx4_dequantize(b))
    w = ops.mx4_quantize(_store(_matrix(_rng(6), 600, 600), "bf16")[1])
    ops.mx4_linear(t, w, out=view)
    assert torch.equal(view, ops.mx4_linear(t, w))


# ---- products ----------------------------------------------------------------------------------------------------------------

def _check_product(c, a, b, bf16_out):
    want = a @ b.T
    room = 2.0 ** -23 * a.shape[1] * (np.abs(a) @ np.abs(b).T)
    if bf16_out:
        room = room + BF16_TOL * np.abs(want)
    assert (np.abs(c - want) <= room).all()


SIZES = [(1, 1, 1), (1, 32, 16), (2, 33, 17), (16, 512, 64), (17, 500, 100), (33, 777, 130), (64, 1024, 15), (65, 256, 63), (66, 257, 65), (128, 100, 128),
         (129, 1500, 300), (300, 4096, 70), (130, 16384, 140), (1000, 777, 1100), (2049, 600, 2050)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_products(n, k, m, out):
    rng = _rng(n, k, m)
    x, xt = _store(_matrix(rng, n, k), "bf16")
    w, wt = _store(0.02 * _matrix(rng, m, k), "bf16")
    a, b = R.rounded(x), R.rounded(w)
    qa, qb = ops.mx4_quantize(xt), ops.mx4_quantize(wt)
    c = ops.mx4_gemm(qa, qb, dtype=DT[out])
    _check_product(c.double().cpu().numpy(), a, b, out == "bf16")
    # the layer quantises the same values to the same bits, and sums are formed in a fixed order
    assert torch.equal(ops.mx4_linear(xt, qb, dtype=DT[out]), c)
    assert torch.equal(ops.mx4_gemm(qa, qb, dtype=DT[out]), c)


@pytest.mark.parametrize("n,k,m", [(1, 4096, 48), (40, 2048, 33), (200, 4096, 200), (513, 1024, 600)])
def test_sums_that_fit_24_bits_are_exact(n, k, m):
    """Values of the grid under scales that differ by up to 2^6: every partial sum is a multiple of 1/4 below 2^22 / 4."""
    rng = _rng(n, k, m, 1)

    def one(rows):
        g = R.GRID[rng.integers(0, 8, (rows, k))] * rng.choice([-1.0, 1.0], (rows, k))
        g[:, ::32] = 6.0                                            # fixes the block's scale
        return g * np.repeat(np.ldexp(1.0, rng.integers(0, 4, (rows, -(-k // 32)))), 32, axis=1)[:, :k]
    a, b = one(n), one(m)
    assert np.array_equal(R.rounded(a), a)
    qa, qb = ops.mx4_quantize(_store(a, "f32")[1]), ops.mx4_quantize(_store(b, "f32")[1])
    assert np.array_equal(ops.mx4_gemm(qa, qb).double().cpu().numpy(), a @ b.T)


@pytest.mark.parametrize("n,k,m", [(3, 700, 40), (70, 300, 201), (300, 512, 130)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_outputs_go_where_they_belong(n, k, m, out):
    """An output with odd rows inside a larger buffer: only its own elements are written."""
    rng = _rng(n, k, m, 2)
    x, w = _store(_matrix(rng, n, k), "f32")[1], ops.mx4_quantize(_store(_matrix(rng, m, k), "f32")[1])
    big = torch.full((n + 4, m + 9), 3.0, device=DEV, dtype=DT[out])
    view = big[1:n + 1, 5:m + 5]
    ops.mx4_linear(x, w, out=view)
    assert torch.equal(view, ops.mx4_linear(x, w, dtype=DT[out]))
    view.fill_(3.0)
    assert bool((big == 3.0).all())


def test_weights_of_a_checkpoint():
    """Buffers laid out on the host are the library's own."""
    w, t = _store(0.02 * _matrix(_rng(8), 100, 700), "f32")
    data, scales = R.packed(*R.quantise(w))
    q = ops.Mx4(torch.from_numpy(data).to(DEV), torch.from_numpy(scales).to(DEV), 100, 700)
    x = _store(_matrix(_rng(9), 5, 700), "bf16")[1]
    assert torch.equal(ops.mx4_linear(x, q), ops.mx4_linear(x, ops.mx4_quantize(t)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,m", [(1, 40, 33), (20, 100, 64), (100, 333, 257), (500, 256, 70), (600, 777, 1100)])
def test_gradients(n, k, m, dtype):
    rng = _rng(n, k, m, 3)
    x, xt = _store(_matrix(rng, n, k), dtype)
    w, wt = _store(0.02 * _matrix(rng, m, k), dtype)
    dy = 1e-3 * _matrix(rng, n, m)
    dy[n // 2] = 0.0                                               # a token without a gradient
    dy, dyt = _store(dy, dtype)
    _, qwt = ops.mx4_quantize(wt, both=True)
    _, qxt = ops.mx4_quantize(xt, both=True)
    dx, dw = ops.mx4_linear_backward(dyt, qwt, qxt)
    assert dx.dtype == DT[dtype] and dw.dtype == torch.float32
    _check_product(dx.double().cpu().numpy(), R.rounded(dy), R.rounded(w.T), dtype == "bf16")
    _check_product(dw.double().cpu().numpy(), R.rounded(dy.T), R.rounded(x.T), False)
    one, none = ops.mx4_linear_backward(dyt, qwt, None)
    assert none is None and torch.equal(one, dx)
    none, one = ops.mx4_linear_backward(dyt, None, qxt)
    assert none is None and torch.equal(one, dw)


# tiles of 64 and of 128 in one launch for both gradients, and pairs that do not go together (other tiles, shared ranges, too many)
@pytest.mark.parametrize("n,k,m", [(65, 1, 65), (130, 70, 1000), (2100, 1400, 2100), (2048, 4096, 80), (4096, 100, 4096)])
def test_gradients_side_by_side(n, k, m):
    x, w, dy = (torch.randn(*s, device=DEV, dtype=torch.bfloat16) for s in ((n, k), (m, k), (n, m)))
    _, qwt = ops.mx4_quantize(w, both=True)
    _, qxt = ops.mx4_quantize(x, both=True)
    dx, dw = ops.mx4_linear_backward(dy, qwt, qxt)
    q, qt = ops.mx4_quantize(dy, both=True)
    assert torch.equal(dx, ops.mx4_gemm(q, qwt, dtype=torch.bfloat16)) and torch.equal(dw, ops.mx4_gemm(qt, qxt, dtype=torch.float32))
    assert bool(dx.isfinite().all()) and float(dx.float().norm()) > 0 and float(dw.norm()) > 0


def test_gradients_by_differences():
    """Operands that the format holds exactly in both directions (magnitudes 1 to 6 of one scale): the loss
    <dy, x w^T> is then linear, and its differences along a direction that stays on the grid are the gradients'."""
    n, k, m = 96, 64, 160
    rng = _rng(10)
    pick = lambda r, c: rng.choice([1.0, 2.0, 3.0, 4.0, 6.0], (r, c)) * rng.choice([-1.0, 1.0], (r, c))  # noqa: E731

    def pin(v):                         # one value of 6 in every block of either direction
        i, j = np.indices(v.shape)
        return np.where((i - j) % 32 == 0, 6.0, v)
    x, w, dy = pin(pick(n, k)), pin(pick(m, k)), pin(pick(n, m))
    step_x, step_w = x.copy(), w.copy()
    step_x[x == 3.0], step_w[w == 3.0] = 4.0, 4.0                   # a step from one grid value to the next
    to = lambda v: _store(v, "f32")[1]  # noqa: E731

    def loss(xv, wv):
        y = ops.mx4_linear(to(xv), ops.mx4_quantize(to(wv)))
        return float((y.double() * torch.from_numpy(dy).to(DEV)).sum())
    dx, dw = ops.mx4_linear_backward(to(dy), ops.mx4_quantize(to(w), both=True)[1], ops.mx4_quantize(to(x), both=True)[1])
    base = loss(x, w)
    assert loss(step_x, w) - base == float((dx.double().cpu().numpy() * (step_x - x)).sum())
    assert loss(x, step_w) - base == float((dw.double().cpu().numpy() * (step_w - w)).sum())


def test_no_tokens():
    w = ops.mx4_quantize(torch.zeros(20, 64, device=DEV))
    assert ops.mx4_linear(torch.zeros(0, 64, device=DEV), w).shape == (0, 20)


def test_products_refuse_mismatched_operands():
    a, b = ops.mx4_quantize(torch.zeros(20, 64, device=DEV)), ops.mx4_quantize(torch.zeros(20, 65, device=DEV))
    x = torch.zeros(3, 64, device=DEV)
    bad = [lambda: ops.mx4_gemm(a, b), lambda: ops.mx4_linear(x, b), lambda: ops.mx4_linear(x.double(), a), lambda: ops.mx4_linear(x, x),
           lambda: ops.mx4_linear(x, a, dtype=torch.float16), lambda: ops.mx4_gemm(a, a, out=torch.empty(3, 3, device=DEV)),
           lambda: ops.mx4_linear_backward(x, None, None), lambda: ops.mx4_linear_backward(x, b, None), lambda: ops.mx4_quantize(x[None]),
           lambda: ops.mx4_quantize(torch.zeros(0, 5, device=DEV)), lambda: ops.Mx4(a.data, a.scales, 21, 64), lambda: ops.Mx4(a.data, a.scales, 20, 600)]
    for f in bad:
        with pytest.raises(gecc.GeccError):
            f()


# ---- the orthogonalised update -------------------------------------------------------------------------------------------------

COEF = (3.4445, -4.7750, 2.0315)


def _gradient(rng, rows, cols, kind):
    if kind == "noise":
        return rng.standard_normal((rows, cols))
    r = min(16, rows, cols)
    low = rng.standard_normal((rows, r)) @ rng.standard_normal((r, cols))
    if kind == "rank":
        return low
    return low + 0.3 * rng.standard_normal((rows, cols))


def _orth_check(o, want, out):
    o = o.double().cpu().numpy()
    assert np.isfinite(o).all()
    off = np.linalg.norm(o - want) / np.linalg.norm(want)
    assert off <= ORTH_TOL + (ORTH_BF16 if out == "bf16" else 0.0), off


@pytest.mark.parametrize("kind", ["noise", "spiked", "rank"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 100), (100, 1), (16, 16), (33, 65), (64, 64), (65, 64), (128, 128), (127, 129), (129, 130), (200, 776), (776, 200),
                                       (300, 301), (512, 512), (900, 130), (1, 300), (5, 700), (16, 257), (17, 1000), (40, 2049), (64, 600), (1000, 33), (700, 64)])
def test_orthogonalised(rows, cols, kind):
    rng = _rng(rows, cols, 4)
    g, t = _store(1e-3 * _gradient(rng, rows, cols, kind), "bf16")
    want, _ = R.orthogonalise(g, None, 0.0, True, 5, COEF, 1e-7, 0.7)
    _orth_check(ops.orthogonalize(t, scale=0.7), want, "bf16")
    _orth_check(ops.orthogonalize(t, scale=0.7, dtype=torch.float32), want, "f32")


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(40, 100), (257, 300), (600, 200), (30, 1000), (555, 60)])
def test_momentum(rows, cols, dtype, nesterov):
    rng = _rng(rows, cols, 5)
    m = torch.zeros(rows, cols, device=DEV)
    ref = np.zeros((rows, cols))
    for _ in range(3):
        g, t = _store(_gradient(rng, rows, cols, "spiked"), dtype)
        o = ops.orthogonalize(t, momentum=m, mu=0.9, nesterov=nesterov)
        want, ref = R.orthogonalise(g, ref, float(np.float32(0.9)), nesterov, 5, COEF, 1e-7, 1.0)
        _orth_check(o, want, "bf16")
        assert np.abs(m.double().cpu().numpy() - ref).max() <= 3 * 2.0 ** -24 * np.abs(ref).max()     # a rounding a step


@pytest.mark.parametrize("batch,rows,cols", [(3, 40, 100), (5, 128, 128), (7, 200, 70), (2, 600, 513), (40, 64, 64), (3, 20, 700), (9, 500, 64)])
def test_batches_are_their_items(batch, rows, cols):
    rng = _rng(batch, rows, cols, 6)
    g = _store(_gradient(rng, batch * rows, cols, "spiked").reshape(batch, rows, cols), "f32")[1]
    m = torch.randn(batch, rows, cols, device=DEV)
    alone = [m[i].clone() for i in range(batch)]
    o = ops.orthogonalize(g, momentum=m)
    for i in range(batch):
        one = ops.orthogonalize(g[i], momentum=alone[i])
        assert torch.equal(alone[i], m[i])
        want, _ = R.orthogonalise(g[i].cpu().numpy(), (alone[i] - g[i]).cpu().numpy() / 0.95, 0.95, True, 5, COEF, 1e-7, 1.0)
        for x in (o[i], one):                       # (a batch may be computed in other tiles than one matrix)
            _orth_check(x, want, "bf16")


@pytest.mark.parametrize("steps", [0, 1, 2, 16])
@pytest.mark.parametrize("rows,cols", [(50, 90), (300, 140), (40, 400)])
def test_numbers_of_steps(rows, cols, steps):
    """Coefficients whose polynomial has 1 as a fixed point of slope 0, so that more steps do not add error: 15 s / 8 ..."""
    rng = _rng(rows, cols, steps)
    g, t = _store(_gradient(rng, rows, cols, "noise"), "f32")
    coef = (1.875, -1.25, 0.375)
    want, _ = R.orthogonalise(g, None, 0, True, steps, coef, 1e-7, 2.0)
    _orth_check(ops.orthogonalize(t, steps=steps, coefficients=coef, scale=2.0, dtype=torch.float32), want, "f32")


@pytest.mark.parametrize("power", [-60, 0, 60])
def test_any_magnitude(power):
    """Squares of such values leave the range of fp32; their norm does not."""
    g, t = _store(np.ldexp(_gradient(_rng(11), 100, 200, "noise"), power), "f32")
    eps = 1e-30
    want, _ = R.orthogonalise(g, None, 0, True, 5, COEF, eps, 1.0)
    _orth_check(ops.orthogonalize(t, eps=eps), want, "bf16")


def test_nothing_to_orthogonalise_and_no_number():
    z = torch.zeros(3, 70, 90, device=DEV)
    z[1] = torch.randn(70, 90, device=DEV)
    z[2] = z[1]
    z[2, 5, 6] = float("nan")
    o = ops.orthogonalize(z).float()
    assert bool((o[0] == 0).all()) and bool(torch.isfinite(o[1]).all()) and bool(torch.isnan(o[2]).all())


def test_strided_gradients_momenta_and_outputs():
    rng = _rng(12)
    for rows, cols in ((70, 131), (300, 90), (20, 501), (333, 50)):
        g = _store(_gradient(rng, rows, cols, "spiked"), "bf16")[1]
        big_g = torch.full((rows, cols + 13), float("nan"), device=DEV, dtype=torch.bfloat16)
        big_m = torch.full((rows, cols + 7), 5.0, device=DEV)
        big_o = torch.full((rows, cols + 3), 5.0, device=DEV, dtype=torch.bfloat16)
        vg, vm, vo = big_g[:, 3:cols + 3], big_m[:, 2:cols + 2], big_o[:, 1:cols + 1]
        vg.copy_(g)
        vm.zero_()
        m = torch.zeros(rows, cols, device=DEV)
        want = ops.orthogonalize(g, momentum=m)
        ops.orthogonalize(vg, momentum=vm, out=vo)
        assert torch.equal(vo, want) and torch.equal(vm, m)
        vm.fill_(5.0), vo.fill_(5.0)
        assert bool((big_m == 5.0).all()) and bool((big_o == 5.0).all())


# sides of up to 64: all steps in fp32, the last of them, from one step to more than the default
@pytest.mark.parametrize("coef", [COEF, (1.5, -0.5, 0.0)])
@pytest.mark.parametrize("steps", [1, 3, 4, 8])
@pytest.mark.parametrize("rows,cols", [(16, 300), (700, 30), (48, 1000)])
def test_long_side_steps(rows, cols, steps, coef):
    rng = _rng(rows, cols, steps, 18)
    g, t = _store(_gradient(rng, rows, cols, "spiked"), "f32")
    want, _ = R.orthogonalise(g, None, 0, True, steps, coef, 1e-7, 2.0)
    _orth_check(ops.orthogonalize(t, steps=steps, coefficients=coef, scale=2.0, dtype=torch.float32), want, "f32")


# ---- ... of long matrices with a shorter side of 65 to 128: bands of 128 of the long side, a launch a step ----------------------
@pytest.mark.parametrize("kind", ["noise", "spiked", "rank"])
@pytest.mark.parametrize("rows,cols", [(65, 257), (128, 512), (100, 513), (96, 1000), (1001, 127), (700, 66), (128, 4096), (3000, 77)])
def test_bands(rows, cols, kind):
    rng = _rng(rows, cols, 14)
    g, t = _store(1e-3 * _gradient(rng, rows, cols, kind), "bf16")
    want, _ = R.orthogonalise(g, None, 0.0, True, 5, COEF, 1e-7, 0.7)
    _orth_check(ops.orthogonalize(t, scale=0.7), want, "bf16")
    _orth_check(ops.orthogonalize(t, scale=0.7, dtype=torch.float32), want, "f32")


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
@pytest.mark.parametrize("rows,cols", [(90, 300), (2000, 128)])
def test_bands_steps(rows, cols, steps):
    rng = _rng(rows, cols, steps, 15)
    g, t = _store(_gradient(rng, rows, cols, "spiked"), "f32")
    want, _ = R.orthogonalise(g, None, 0, True, steps, COEF, 1e-7, 2.0)
    _orth_check(ops.orthogonalize(t, steps=steps, scale=2.0, dtype=torch.float32), want, "f32")


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(70, 1025), (600, 128)])
def test_bands_momentum(rows, cols, dtype, nesterov):
    rng = _rng(rows, cols, 16)
    m = torch.zeros(rows, cols, device=DEV)
    ref = np.zeros((rows, cols))
    for _ in range(3):
        g, t = _store(_gradient(rng, rows, cols, "spiked"), dtype)
        o = ops.orthogonalize(t, momentum=m, mu=0.9, nesterov=nesterov)
        want, ref = R.orthogonalise(g, ref, float(np.float32(0.9)), nesterov, 5, COEF, 1e-7, 1.0)
        _orth_check(o, want, "bf16")
        assert np.abs(m.double().cpu().numpy() - ref).max() <= 3 * 2.0 ** -24 * np.abs(ref).max()     # a rounding a step


# several bands a workgroup (more than 256 of them), and more items than go through the steps together (about 192 MiB of them)
@pytest.mark.parametrize("batch,rows,cols", [(3, 70, 600), (40, 128, 1500), (300, 66, 400), (1000, 65, 257)])
def test_bands_batches(batch, rows, cols):
    rng = _rng(batch, rows, cols, 17)
    g = torch.from_numpy(rng.standard_normal((batch, rows, cols)).astype(np.float32)).to(DEV)
    kept = g.clone()
    o = ops.orthogonalize(g, dtype=torch.float32)
    assert torch.equal(g, kept)
    for i in sorted({0, 1, batch // 2, batch // 2 + 1, batch - 2, batch - 1}):
        want, _ = R.orthogonalise(g[i].double().cpu().numpy(), None, 0.0, True, 5, COEF, 1e-7, 1.0)
        _orth_check(o[i], want, "f32")
    # S = X X^T after the steps has a trace of about the rank: none of the items between was left out
    trace = o.square().sum((1, 2))
    assert bool((trace > 0.4 * min(rows, cols)).all()) and bool((trace < 1.6 * min(rows, cols)).all())


@pytest.mark.parametrize("rows,cols", [(80, 290), (290, 80)])
def test_bands_strides_zeros_and_no_number(rows, cols):
    big = torch.randn(2, rows + 3, cols + 5, device=DEV)
    m0 = torch.randn(2, rows + 1, cols + 2, device=DEV)
    g, m = big[:, 1:rows + 1, 3:cols + 3], m0[:, :rows, 1:cols + 1]
    out = torch.full((2, rows + 2, cols + 7), 7.0, device=DEV)
    dense_m = m.contiguous()
    want = ops.orthogonalize(g.contiguous(), momentum=dense_m, dtype=torch.float32)
    before = m0.clone()
    ops.orthogonalize(g, momentum=m, out=out[:, 2:, 1:cols + 1])
    torch.testing.assert_close(out[:, 2:, 1:cols + 1], want, rtol=0, atol=1e-5)      # (another order of the norm's sum)
    assert torch.equal(m, dense_m)
    out[:, 2:, 1:cols + 1] = 7.0
    assert bool((out == 7.0).all())
    m0[:, :rows, 1:cols + 1] = before[:, :rows, 1:cols + 1]
    assert torch.equal(m0, before)
    z = torch.zeros(2, rows, cols, device=DEV)
    z[1, 3, 4] = float("nan")
    o = ops.orthogonalize(z, dtype=torch.float32)
    assert bool((o[0] == 0).all()) and bool(o[1].isnan().all())


def test_orthogonalize_refuses():
    g = torch.zeros(4, 6, device=DEV)
    for f in (lambda: ops.orthogonalize(g.double()), lambda: ops.orthogonalize(g[0]), lambda: ops.orthogonalize(g, momentum=g.bfloat16()),
              lambda: ops.orthogonalize(g, momentum=torch.zeros(6, 4, device=DEV)), lambda: ops.orthogonalize(g, momentum=torch.zeros(6, 4, device=DEV).t()),
              lambda: ops.orthogonalize(g, out=torch.empty(6, 4, device=DEV)), lambda: ops.orthogonalize(g, steps=17),
              lambda: ops.orthogonalize(g, eps=0.0), lambda: ops.orthogonalize(g, coefficients=(50.0, 0.0, 0.0)), lambda: ops.orthogonalize(g, dtype=torch.float16),
              lambda: ops.orthogonalize(torch.zeros(0, 6, device=DEV))):
        with pytest.raises(gecc.GeccError):
            f()


# ---- streams and graphs --------------------------------------------------------------------------------------------------------

def _step(x, w, dy, m):
    """One pass through everything."""
    q, qt = ops.mx4_quantize(w, both=True)
    xq, xt = ops.mx4_quantize(x, both=True)
    y = ops.mx4_gemm(xq, q)
    dx, dw = ops.mx4_linear_backward(dy, qt, xt)
    return y, dx, dw, ops.orthogonalize(dw, momentum=m), ops.mx4_linear(x[:2], q)


def _step_inputs():
    rng = _rng(13)
    return [_store(_matrix(rng, *s), "f32")[1] for s in ((300, 200), (150, 200), (300, 150))]


def test_on_another_stream():
    x, w, dy = _step_inputs()
    m0, m1 = torch.zeros(150, 200, device=DEV), torch.zeros(150, 200, device=DEV)
    want = _step(x, w, dy, m0)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = _step(x, w, dy, m1)
    st.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert torch.equal(m0, m1)


def test_in_a_graph():
    x, w, dy = _step_inputs()
    m, m_ref = torch.zeros(150, 200, device=DEV), torch.zeros(150, 200, device=DEV)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        _step(x, w, dy, torch.zeros(150, 200, device=DEV))
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(x, w, dy, m)
    m.zero_()
    for i in range(4):
        x.mul_(-0.5 if i % 2 else 1.5)
        want = _step(x, w, dy, m_ref)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b), i
        assert torch.equal(m, m_ref)


# ---- together ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("protect", [False, True])
def test_a_layer_learns(protect):
    """The example: the loss at least halves (a layer that did not learn would keep it), the protected gradients report no
    errors, and a token served from packed weights gets what the batch gets."""
    from paper_2508_04355_amd import train_layer
    losses, status, layers = train_layer.train(steps=60, tokens=256, width=128, hidden=200, protect=protect)
    assert np.isfinite(losses).all() and losses[-1] < losses[0] / 2
    assert status == gecc.CLEAN
    x = torch.randn(70, 128, device=DEV)
    h = torch.relu(ops.mx4_gemm(ops.mx4_quantize(x), ops.mx4_quantize(layers[0].w)))
    y = ops.mx4_gemm(ops.mx4_quantize(h), ops.mx4_quantize(layers[1].w))
    for i in (0, 33, 69):
        # (the fp32 sums of one row may be formed in another order: half an ulp at their size, then quantised again)
        one = train_layer.serve(layers, x[i:i + 1])
        assert float((one - y[i]).norm() / y[i].norm()) < 0.02
