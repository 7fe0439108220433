"""CPU-side checks of the operators' C ABI (include/gecc_ops.h) and of their binding: exported symbols, struct layout, buffer
sizes, and refusals, none of which touches a GPU."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import ops_reference as R
from paper_2508_04355_amd import build as build_mod
from paper_2508_04355_amd import gecc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, WORKSPACE, ALIGN = -1, -2, -4
OK, ODD = C.c_void_p(1 << 16), C.c_void_p((1 << 16) + 1)


@pytest.fixture(scope="module")
def ops():
    if not os.path.exists(gecc._LIB_PATH):
        build_mod.build(verbose=False)
    from paper_2508_04355_amd import ops
    ops.lib()
    return ops


def test_every_declared_symbol_is_exported(ops):
    header = open(os.path.join(ROOT, "include", "gecc_ops.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(gecc_[a-z0-9_]+)\s*\(", header))
    assert declared == set(ops._SYMBOLS)
    L = C.CDLL(gecc._LIB_PATH)
    for name in declared:
        assert hasattr(L, name), name


def test_struct_layout_matches_the_header(ops):
    assert C.sizeof(ops.OrthParams) == 8 * 4 + 6 * 8 + 6 * 4


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 256), (15, 257), (16, 512), (17, 513), (1000, 777), (16384, 4096)])
def test_buffer_sizes(ops, rows, cols):
    L = ops.lib()
    if rows * cols < 1 << 20:
        data, scales = R.packed(*R.quantise(np.zeros((rows, cols))))
        assert (L.gecc_mx4_data_bytes(rows, cols), L.gecc_mx4_scale_bytes(rows, cols)) == (data.size, scales.size)
    else:
        assert L.gecc_mx4_data_bytes(rows, cols) == rows * cols // 2
        assert L.gecc_mx4_scale_bytes(rows, cols) == rows * cols // 32
    for bad in ((0, cols), (rows, 0), (-1, cols), (rows, (1 << 24) + 1)):
        assert L.gecc_mx4_data_bytes(*bad) == 0 and L.gecc_mx4_scale_bytes(*bad) == 0


def test_quantize_and_dequantize_refuse(ops):
    L = ops.lib()
    good = [OK, 0, 3, 100, 100, OK, OK, OK, OK, None]

    def call(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return L.gecc_mx4_quantize(*a)
    for kw in (dict(_0=None), dict(_1=2), dict(_2=0), dict(_3=0), dict(_3=-5), dict(_4=99), dict(_5=None), dict(_6=None), dict(_7=None),
               dict(_8=None), dict(_5=None, _6=None, _7=None, _8=None), dict(_2=(1 << 24) + 1, _4=1 << 25)):
        assert call(**kw) == ARG, kw
    for kw in (dict(_0=C.c_void_p((1 << 16) + 2)), dict(_5=ODD), dict(_6=ODD), dict(_7=ODD), dict(_8=ODD)):
        assert call(**kw) == ALIGN, kw
    assert L.gecc_mx4_dequantize(None, OK, 3, 100, OK, 0, 100, None) == ARG
    assert L.gecc_mx4_dequantize(OK, OK, 3, 100, OK, 0, 99, None) == ARG
    assert L.gecc_mx4_dequantize(OK, OK, 3, 100, OK, 5, 100, None) == ARG
    assert L.gecc_mx4_dequantize(OK, OK, 0, 100, OK, 0, 100, None) == ARG
    assert L.gecc_mx4_dequantize(ODD, OK, 3, 100, OK, 0, 100, None) == ALIGN
    assert L.gecc_mx4_dequantize(OK, OK, 3, 100, ODD, 1, 100, None) == ALIGN


def test_products_refuse(ops):
    L = ops.lib()
    n, k, m = 200, 16384, 200
    need = L.gecc_mx4_gemm_workspace(n, k, m)
    assert need > 0                                     # few tiles: k is shared out
    gemm = [n, k, m, OK, OK, OK, OK, OK, 0, m, OK, need, None]
    lin = [n, k, m, OK, 1, k, OK, OK, OK, 1, m, OK, L.gecc_mx4_linear_workspace(n, k, m), None]
    back = [n, k, m, OK, 1, m, OK, OK, OK, OK, OK, 1, k, OK, k, OK, L.gecc_mx4_linear_backward_workspace(n, k, m), None]

    def each(f, good, bads, code):
        for bad in bads:
            a = list(good)
            for pos, v in bad.items():
                a[pos] = v
            assert f(*a) == code, (f.__name__, bad)
    each(L.gecc_mx4_gemm, gemm, [{0: 0}, {1: -1}, {2: 0}, {3: None}, {4: None}, {5: None}, {6: None}, {7: None}, {8: 9}, {9: m - 1}], ARG)
    each(L.gecc_mx4_gemm, gemm, [{3: ODD}, {4: ODD}, {5: ODD}, {6: ODD}, {7: ODD}, {10: ODD}], ALIGN)
    each(L.gecc_mx4_gemm, gemm, [{10: None}, {11: need - 1}], WORKSPACE)
    each(L.gecc_mx4_linear, lin, [{0: 0}, {3: None}, {4: 3}, {5: k - 1}, {6: None}, {7: None}, {8: None}, {9: -1}, {10: m - 1}], ARG)
    each(L.gecc_mx4_linear, lin, [{3: ODD}, {6: ODD}, {7: ODD}, {8: ODD}, {11: ODD}], ALIGN)
    each(L.gecc_mx4_linear, lin, [{11: None}, {12: lin[12] - 1}], WORKSPACE)
    each(L.gecc_mx4_linear_backward, back, [{0: 0}, {3: None}, {4: 7}, {5: m - 1}, {6: None}, {7: None}, {8: None}, {9: None}, {11: 5}, {12: k - 1},
                                            {14: k - 1}, {10: None, 13: None}], ARG)
    each(L.gecc_mx4_linear_backward, back, [{3: ODD}, {6: ODD}, {9: ODD}, {10: ODD}, {13: C.c_void_p((1 << 16) + 2)}, {15: ODD}], ALIGN)
    each(L.gecc_mx4_linear_backward, back, [{15: None}, {16: back[16] - 1}], WORKSPACE)
    assert L.gecc_mx4_linear_workspace(1, 4096, 14336) == 0     # one token needs none


def _orth(ops, **kw):
    d = dict(rows=160, cols=300, batch=1, dtype=0, out_dtype=1, steps=5, nesterov=1, reserved=0, ld_g=300, ld_m=300, ld_o=300, stride_g=0,
             stride_m=0, stride_o=0, mu=0.95, eps=1e-7, scale=1.0, a=3.4445, b=-4.775, c=2.0315)
    d.update(kw)
    return ops.OrthParams(**d)


def test_orthogonalize_refuses(ops):
    L = ops.lib()
    p = _orth(ops)
    need = L.gecc_orthogonalize_workspace(C.byref(p))
    assert need > 0
    small = _orth(ops, rows=128, cols=256, ld_g=256, ld_m=256, ld_o=256)
    assert L.gecc_orthogonalize_workspace(C.byref(small)) == 0      # (one launch, no workspace)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(rows=0), dict(cols=-1), dict(batch=0), dict(batch=65536), dict(dtype=2), dict(out_dtype=-1), dict(steps=-1), dict(steps=17),
                dict(nesterov=2), dict(reserved=1), dict(mu=nan), dict(eps=0.0), dict(eps=inf), dict(scale=inf), dict(a=nan), dict(b=inf),
                dict(a=100.0), dict(c=1e30), dict(rows=(1 << 24) + 1)):
        q = _orth(ops, **bad)
        assert L.gecc_orthogonalize_workspace(C.byref(q)) == 0, bad
        assert L.gecc_orthogonalize(C.byref(q), OK, OK, OK, OK, need, None) == ARG, bad
    for bad in (dict(ld_g=299), dict(ld_m=299), dict(ld_o=299), dict(batch=2), dict(batch=2, stride_g=48000, stride_o=48000, stride_m=47999)):
        q = _orth(ops, **bad)
        assert L.gecc_orthogonalize(C.byref(q), OK, OK, OK, OK, 1 << 30, None) == ARG, bad
    assert L.gecc_orthogonalize(None, OK, OK, OK, OK, need, None) == ARG
    assert L.gecc_orthogonalize(C.byref(p), None, OK, OK, OK, need, None) == ARG
    assert L.gecc_orthogonalize(C.byref(p), OK, OK, None, OK, need, None) == ARG
    assert L.gecc_orthogonalize(C.byref(p), ODD, OK, OK, OK, need, None) == ALIGN
    assert L.gecc_orthogonalize(C.byref(p), OK, C.c_void_p((1 << 16) + 2), OK, OK, need, None) == ALIGN
    assert L.gecc_orthogonalize(C.byref(p), OK, OK, OK, ODD, need, None) == ALIGN
    assert L.gecc_orthogonalize(C.byref(p), OK, OK, OK, None, need, None) == WORKSPACE
    assert L.gecc_orthogonalize(C.byref(p), OK, OK, OK, OK, need - 1, None) == WORKSPACE
    # a momentum buffer that is not there needs no leading dimension
    q = _orth(ops, ld_m=0)
    assert L.gecc_orthogonalize(C.byref(q), OK, OK, OK, OK, need, None) == ARG


def test_the_binding_refuses_what_is_not_on_the_gpu(ops):
    x = torch.zeros(4, 32)
    for f in (lambda: ops.mx4_quantize(x), lambda: ops.mx4_linear(x, None), lambda: ops.orthogonalize(x),
              lambda: ops.mx4_linear_backward(x, None, None), lambda: ops.Mx4(x, x, 4, 32), lambda: ops.mx4_dequantize(x),
              lambda: ops.mx4_gemm(x, x)):
        with pytest.raises(gecc.GeccError):
            f()


def test_the_reference_rounds_as_the_format_says():
    """Every tie of the grid at a scale of one (a block whose largest value is 4), and the ends."""
    x = np.zeros((1, 32))
    x[0, :12] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, 6.9, 7.9]
    codes, scales = R.quantise(x)
    assert scales[0, 0] == 127
    assert R.values(codes, scales)[0, :12].tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.0, -1.0, 6.0, 6.0]
