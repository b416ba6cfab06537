"""CPU checks of the residual-block operators' ABI: struct layouts against the C compiler, workspace sizing, and every
refusal that the header names (all of them on the host: nothing here launches a kernel)."""
import ctypes
import os
import subprocess

import pytest

import paper_1811_12843_amd as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # a placeholder address, 256-byte aligned


def mat(cols, rows=4, p=P, ld=None, cell=None):
    ld = cols if ld is None else ld
    return L.lipz_mat(p, ld, rows * ld if cell is None else cell)


def norm(**kw):
    d = dict(dtype=L.LIPZ_BF16, y_dtype=L.LIPZ_BF16, cells=2, rows=4, cols=24, eps=1e-5, x=mat(24), residual=mat(24),
             h=mat(24), y=mat(24), gamma=P, gamma_cell=24, rstd=P, y_scale=P)
    return L.lipz_rms_norm_args(**dict(d, **kw))


def norm_bwd(**kw):
    d = dict(dtype=L.LIPZ_BF16, cells=2, rows=4, cols=24, h=mat(24), dy=mat(24), dh=mat(24), dx=mat(24), gamma=P,
             gamma_cell=24, rstd=P, dgamma=P, dgamma_cell=24)
    return L.lipz_rms_norm_backward_args(**dict(d, **kw))


NONE = L.lipz_mat()


def linear(**kw):
    d = dict(dtype=L.LIPZ_BF16, cells=2, rows=4, fan_in=24, fan_out=40, act=L.LIPZ_ACT_LRELU, slope=0.2, x=mat(24),
             w=mat(40, 24), residual=mat(40), pre=mat(40), y=mat(40), bias=P, bias_cell=40)
    return L.lipz_linear_args(**dict(d, **kw))


def linear_bwd(**kw):
    d = dict(dtype=L.LIPZ_BF16, cells=2, rows=4, fan_in=24, fan_out=40, act=L.LIPZ_ACT_SILU, slope=0.2, x=mat(24),
             w=mat(40, 24), pre=mat(40), dy=mat(40), dx=mat(24), dw=mat(40, 24), db=P, db_cell=40)
    return L.lipz_linear_backward_args(**dict(d, **kw))


def quant(**kw):
    d = dict(dtype=L.LIPZ_BF16, cells=2, fan_in=24, fan_out=40, w=mat(40, 24), q=mat(24, 40), scale=P, scale_cell=40)
    return L.lipz_quantize_weights_args(**dict(d, **kw))


def linear_fp8(**kw):
    d = dict(y_dtype=L.LIPZ_BF16, cells=2, rows=4, fan_in=24, fan_out=40, act=L.LIPZ_ACT_GELU, slope=0.2, x=mat(24),
             w=mat(24, 40), residual=mat(40), y=mat(40), x_scale=P, x_scale_cell=4, w_scale=P, w_scale_cell=40, bias=P,
             bias_cell=40)
    return L.lipz_linear_fp8_args(**dict(d, **kw))


BAD = {
    "lipz_rms_norm": (norm, [
        dict(dtype=3), dict(dtype=-1), dict(y_dtype=L.LIPZ_F32), dict(cells=0), dict(rows=-1), dict(cols=0), dict(eps=0.0),
        dict(eps=float("nan")), dict(eps=float("inf")), dict(x=NONE), dict(y=NONE), dict(gamma=None),
        dict(y_dtype=L.LIPZ_FP8, y_scale=None), dict(x=mat(24, ld=23)), dict(y=mat(24, cell=-1)), dict(x=mat(24, p=P + 1)),
        dict(y=mat(24, cell=95)), dict(h=mat(24, cell=0)), dict(gamma=P + 2), dict(rstd=P + 2), dict(gamma_cell=-24)], [
        dict(cols=(1 << 20) + 1, x=mat((1 << 20) + 1), residual=NONE, h=NONE, y=mat((1 << 20) + 1)),
        dict(x=mat(24, ld=(1 << 20) + 8)), dict(cells=65536)]),
    "lipz_rms_norm_backward": (norm_bwd, [
        dict(dtype=3), dict(cells=0), dict(rows=-1), dict(cols=0), dict(h=NONE), dict(dy=NONE), dict(dx=NONE),
        dict(gamma=None), dict(rstd=None), dict(rstd=P + 1), dict(dy=mat(24, ld=8)), dict(dx=mat(24, cell=24)),
        dict(dgamma_cell=23), dict(dgamma=P + 1)], [
        dict(dh=mat(24, ld=(1 << 20) + 8)), dict(cells=65536)]),
    "lipz_linear": (linear, [
        dict(dtype=3), dict(cells=0), dict(rows=-1), dict(fan_in=0), dict(fan_out=0), dict(act=6), dict(act=-1),
        dict(slope=0.0), dict(slope=float("inf")), dict(x=NONE), dict(w=NONE), dict(y=NONE), dict(x=mat(23)),
        dict(w=mat(39, 24)), dict(y=mat(40, cell=40)), dict(pre=mat(40, p=P + 1)), dict(residual=mat(40, cell=-1)),
        dict(bias=P + 2), dict(bias_cell=-1)], [
        dict(cells=65536), dict(rows=(1 << 21) + 1), dict(fan_in=(1 << 20) + 1), dict(x=mat(24, ld=(1 << 20) + 2)),
        dict(rows=1 << 21, fan_out=1 << 20, w=mat(1 << 20, 24), residual=NONE, pre=NONE, y=mat(1 << 20, 1 << 21))]),
    "lipz_linear_backward": (linear_bwd, [
        dict(dtype=3), dict(cells=0), dict(rows=-1), dict(fan_in=0), dict(fan_out=0), dict(act=7), dict(pre=NONE),
        dict(dy=NONE), dict(x=NONE), dict(w=NONE), dict(dx=NONE, dw=NONE, db=None), dict(dx=mat(24, cell=24)),
        dict(dw=mat(40, 24, cell=0)), dict(db_cell=39), dict(act=L.LIPZ_ACT_LRELU, slope=-1.0), dict(dy=mat(39))], [
        dict(cells=65536), dict(rows=(1 << 21) + 1), dict(w=mat(40, 24, ld=(1 << 20) + 2))]),
    "lipz_quantize_weights": (quant, [
        dict(dtype=3), dict(cells=0), dict(fan_in=0), dict(fan_out=0), dict(w=NONE), dict(q=NONE), dict(scale=None),
        dict(q=mat(23, 40)), dict(q=mat(24, 40, cell=24)), dict(scale_cell=39), dict(scale=P + 1)], [
        dict(cells=65536), dict(fan_out=(1 << 20) + 1)]),
    "lipz_linear_fp8": (linear_fp8, [
        dict(y_dtype=3), dict(cells=0), dict(rows=-1), dict(fan_in=0), dict(fan_out=0), dict(act=6), dict(x=NONE),
        dict(w=NONE), dict(y=NONE), dict(x_scale=None), dict(w_scale=None), dict(w=mat(23, 40)), dict(y=mat(40, cell=39)),
        dict(x_scale=P + 1), dict(x_scale_cell=-4)], [
        dict(cells=65536), dict(rows=(1 << 21) + 1)]),
}


@pytest.mark.parametrize("name", sorted(BAD))
def test_refusals(name):
    make, bad, unsupported = BAD[name]
    fn, need = getattr(L, name), getattr(L, name + "_workspace_bytes")
    nb = need(make())
    assert nb > 0 and nb % 256 == 0
    for kws, status in ((bad, L.LIPZ_E_INVAL), (unsupported, L.LIPZ_E_UNSUPPORTED)):
        for kw in kws:
            a = make(**kw)
            assert need(a) == 0, kw
            with pytest.raises(L.LipzError) as e:
                fn(a, P, 1 << 40, None)
            assert e.value.status == status, kw
    a = make()
    a.abi_version = 99
    assert need(a) == 0
    for p, n in ((None, nb), (P + 128, nb), (P, nb - 1)):
        with pytest.raises(L.LipzError) as e:
            fn(make(), p, n, None)
        assert e.value.status == L.LIPZ_E_WORKSPACE
    lib = L.load_library()
    assert getattr(lib, name)(None, P, nb, None) == L.LIPZ_E_INVAL
    assert getattr(lib, name + "_workspace_bytes")(None) == 0


@pytest.mark.parametrize("make,name,kw", [
    (norm, "lipz_rms_norm", dict(y=L.lipz_mat(P, 48, 24), x=L.lipz_mat(P, 48, 24))),
    (norm, "lipz_rms_norm", dict(x=mat(24, cell=0), gamma_cell=0)),
    (norm_bwd, "lipz_rms_norm_backward", dict(dx=L.lipz_mat(P, 48, 24), dy=L.lipz_mat(P, 48, 24))),
    (norm_bwd, "lipz_rms_norm_backward", dict(h=mat(24, cell=0), gamma_cell=0)),
    (linear, "lipz_linear", dict(y=L.lipz_mat(P, 80, 40), x=mat(24, cell=0), w=mat(40, 24, cell=0), bias_cell=0)),
    (linear_bwd, "lipz_linear_backward", dict(act=L.LIPZ_ACT_LINEAR, pre=NONE)),
    (linear_bwd, "lipz_linear_backward", dict(dx=NONE, w=NONE)),
    (linear_bwd, "lipz_linear_backward", dict(dw=NONE, x=NONE, db=None)),
    (linear_fp8, "lipz_linear_fp8", dict(x=mat(24, cell=0), w_scale_cell=0, bias=None, residual=NONE))])
def test_cells_inside_rows_shared_inputs_and_left_out_ones_are_taken(make, name, kw):
    """Cells side by side in a row, inputs shared by the cells, optional matrices left out."""
    assert getattr(L, name + "_workspace_bytes")(make(**kw)) > 0


@pytest.mark.parametrize("name", ["lipz_mat"] + [n + "_args" for n in sorted(BAD)])
def test_struct_layout_matches_c(name, tmp_path):
    cls = getattr(L, name)
    fields = [f for f, _ in cls._fields_]
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "lipz.h"', "int main(void) {",
           f'printf("%zu\\n", sizeof({name}));']
    src += [f'printf("%zu\\n", offsetof({name}, {f}));' for f in fields]
    (tmp_path / "t.c").write_text("\n".join(src + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")],
                   check=True)
    out = [int(x) for x in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True,
                                          check=True).stdout.split()]
    assert out[0] == ctypes.sizeof(cls)
    assert out[1:] == [getattr(cls, f).offset for f in fields]


def test_norms_refuse_rows_whose_index_would_wrap():
    for make, name in ((norm, "lipz_rms_norm"), (norm_bwd, "lipz_rms_norm_backward")):
        far = {f: L.lipz_mat(P, 24, 24 << 31) for f, t in make()._fields_ if t is L.lipz_mat}
        assert getattr(L, name + "_workspace_bytes")(make(rows=1 << 30, **far)) > 0
        for rows in ((1 << 30) + 1, (1 << 31) - 1):
            a = make(rows=rows, **far)
            assert getattr(L, name + "_workspace_bytes")(a) == 0
            with pytest.raises(L.LipzError) as e:
                getattr(L, name)(a, P, 1 << 40, None)
            assert e.value.status == L.LIPZ_E_UNSUPPORTED
