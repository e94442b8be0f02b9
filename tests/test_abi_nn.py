"""CPU checks of the feed-forward operators' C ABI and binding: struct layouts,
refusals on the host (nothing is enqueued on these paths) and the workspace sizes."""
import ctypes
import os
import re
import subprocess

import pytest

import paper_1807_11091_amd as sa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # a 256-byte aligned non-null address; never dereferenced on these paths
STRUCTS = {"sa_layer_norm_desc": sa.LayerNormDesc, "sa_layer_norm_bwd_desc": sa.LayerNormBwdDesc,
           "sa_linear_desc": sa.LinearDesc, "sa_linear_bwd_desc": sa.LinearBwdDesc, "sa_glu_desc": sa.GluDesc,
           "sa_glu_bwd_desc": sa.GluBwdDesc}


def test_struct_layouts_match_header(tmp_path):
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "structadmm.h"', "int main(void){"]
    for st, cls in STRUCTS.items():
        lines.append(f'printf("{st} sizeof %zu\\n", sizeof({st}));')
        lines += [f'printf("{st} {f} %zu\\n", offsetof({st}, {f}));' for f, _ in cls._fields_]
    names = {"SA_BF16": sa.BF16, "SA_F16": sa.F16, "SA_F32": sa.F32, "SA_ACT_NONE": sa.ACT_NONE,
             "SA_ACT_RELU": sa.ACT_RELU, "SA_ACT_SIGMOID": sa.ACT_SIGMOID, "SA_ACT_SILU": sa.ACT_SILU,
             "SA_ACT_GELU": sa.ACT_GELU, "SA_ACT_GELU_TANH": sa.ACT_GELU_TANH, "SA_MAX_LD": sa.MAX_LD}
    lines += [f'printf("const {n} %d\\n", (int){n});' for n in names]
    lines.append("return 0;}")
    src, exe = str(tmp_path / "l.c"), str(tmp_path / "l")
    open(src, "w").write("\n".join(lines))
    subprocess.check_call(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                           "/opt/rocm/include", src, "-o", exe])
    got = {}
    for line in subprocess.check_output([exe]).decode().splitlines():
        st, f, v = line.split()
        got[(st, f)] = int(v)
    for st, cls in STRUCTS.items():
        assert ctypes.sizeof(cls) == got[(st, "sizeof")], st
        for f, _ in cls._fields_:
            assert getattr(cls, f).offset == got[(st, f)], (st, f)
    for n, v in names.items():
        assert got[("const", n)] == v, n


def addresses(*names):
    return {n: FAKE * (i + 1) for i, n in enumerate(names)}


GOOD = {
    "layer_norm_fwd": (sa.LayerNormDesc, dict(rows=4, cols=8, type=sa.BF16, eps=1e-5, ldx=8, ldy=8,
                                              **addresses("X", "Y", "gamma", "beta", "mean", "rstd"))),
    "layer_norm_bwd": (sa.LayerNormBwdDesc, dict(rows=4, cols=8, type=sa.F16, lddy=8, ldx=8, lddr=8, lddx=8,
                                                 **addresses("dY", "X", "mean", "rstd", "gamma", "dR", "dX", "dgamma",
                                                             "dbeta"))),
    "linear_fwd": (sa.LinearDesc, dict(M=4, N=16, K=8, type=sa.BF16, out_type=sa.BF16, act=sa.ACT_SILU, ldx=8, ldw=8,
                                       ldr=16, ldy=16, ldz=16, **addresses("X", "W", "bias", "R", "Y", "Z"))),
    "linear_bwd": (sa.LinearBwdDesc, dict(M=4, N=16, K=8, type=sa.BF16, dw_type=sa.F32, act=sa.ACT_SILU, lddy=16,
                                          ldz=16, ldx=8, ldw=8, lddx=8, lddw=8,
                                          **addresses("dY", "Z", "X", "W", "dX", "dW", "dbias"))),
    "glu_fwd": (sa.GluDesc, dict(M=4, N=16, K=8, type=sa.F16, act=sa.ACT_SILU, ldx=8, ldw=8, ldh=16, ldgu=16,
                                 **addresses("X", "Wg", "Wu", "bg", "bu", "H", "G", "U"))),
    "glu_bwd": (sa.GluBwdDesc, dict(M=4, N=16, K=8, type=sa.F16, dw_type=sa.F16, act=sa.ACT_SILU, lddh=16, ldgu=16,
                                    ldx=8, ldw=8, lddx=8, lddw=8,
                                    **addresses("dH", "G", "U", "X", "Wg", "Wu", "dX", "dWg", "dWu", "dbg", "dbu"))),
}


def call(op, **kw):
    cls, good = GOOD[op]
    d = cls(**{**good, **kw})
    rc = getattr(sa.lib(), f"structadmm_{op}")(ctypes.byref(d), None)
    return rc, sa.lib().structadmm_last_error().decode()


REFUSED = [
    ("layer_norm_fwd", dict(rows=-1), -1), ("layer_norm_fwd", dict(cols=0), -1), ("layer_norm_fwd", dict(type=3), -1),
    ("layer_norm_fwd", dict(X=None), -1), ("layer_norm_fwd", dict(Y=None), -1), ("layer_norm_fwd", dict(ldx=7), -1),
    ("layer_norm_fwd", dict(ldy=7), -1), ("layer_norm_fwd", dict(eps=-1.0), -1),
    ("layer_norm_fwd", dict(eps=float("nan")), -1), ("layer_norm_fwd", dict(X=FAKE + 1), -2),
    ("layer_norm_fwd", dict(gamma=FAKE + 2), -2), ("layer_norm_fwd", dict(Y=FAKE, ldy=9), -1),
    ("layer_norm_fwd", dict(ldx=(1 << 21) + 1), -4), ("layer_norm_fwd", dict(rows=1 << 31), -1),
    ("layer_norm_bwd", dict(mean=None), -1), ("layer_norm_bwd", dict(rstd=None), -1),
    ("layer_norm_bwd", dict(dX=None, dgamma=None, dbeta=None), -1), ("layer_norm_bwd", dict(dX=2 * FAKE), -1),
    ("layer_norm_bwd", dict(lddr=7), -1), ("layer_norm_bwd", dict(dY=None), -1), ("layer_norm_bwd", {}, -3),
    ("linear_fwd", dict(M=-1), -1), ("linear_fwd", dict(type=sa.F32), -4), ("linear_fwd", dict(type=9), -1),
    ("linear_fwd", dict(out_type=sa.F16), -1), ("linear_fwd", dict(act=6), -1), ("linear_fwd", dict(act=-1), -1),
    ("linear_fwd", dict(X=None), -1), ("linear_fwd", dict(W=None), -1), ("linear_fwd", dict(Y=None), -1),
    ("linear_fwd", dict(ldx=7), -1), ("linear_fwd", dict(ldw=7), -1), ("linear_fwd", dict(ldr=15), -1),
    ("linear_fwd", dict(ldz=15), -1), ("linear_fwd", dict(W=2 * FAKE + 1), -2), ("linear_fwd", dict(Y=FAKE), -1),
    ("linear_fwd", dict(Y=4 * FAKE, ldy=17), -1), ("linear_fwd", dict(Z=5 * FAKE), -1),
    ("linear_fwd", dict(K=(1 << 21) + 1, ldx=(1 << 21) + 1, ldw=(1 << 21) + 1), -4),
    ("linear_bwd", dict(Z=None), -1), ("linear_bwd", dict(X=None), -1), ("linear_bwd", dict(W=None), -1),
    ("linear_bwd", dict(dX=None, dW=None, dbias=None), -1), ("linear_bwd", dict(dw_type=sa.F16), -1),
    ("linear_bwd", dict(dX=FAKE), -1), ("linear_bwd", dict(dW=4 * FAKE), -1), ("linear_bwd", dict(dW=6 * FAKE + 2), -2),
    ("linear_bwd", {}, -3), ("linear_bwd", dict(ws=FAKE + 16, ws_bytes=1 << 30), -2),
    ("glu_fwd", dict(G=None), -1), ("glu_fwd", dict(Wu=None), -1), ("glu_fwd", dict(H=FAKE), -1),
    ("glu_fwd", dict(U=7 * FAKE), -1), ("glu_fwd", dict(ldgu=15), -1), ("glu_fwd", dict(bg=FAKE + 1), -2),
    ("glu_bwd", dict(dWu=None), -1), ("glu_bwd", dict(U=None), -1), ("glu_bwd", dict(Wg=None), -1),
    ("glu_bwd", dict(dX=None, dWg=None, dWu=None, dbg=None, dbu=None), -1), ("glu_bwd", dict(dX=4 * FAKE), -1),
    ("glu_bwd", dict(lddw=7), -1), ("glu_bwd", {}, -3),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refusals(i):
    op, kw, code = REFUSED[i]
    rc, msg = call(op, **kw)
    assert rc == code, (op, kw, msg)
    assert op in msg


@pytest.mark.parametrize("op", list(GOOD))
def test_null_descriptor(op):
    assert getattr(sa.lib(), f"structadmm_{op}")(None, None) == -1


@pytest.mark.parametrize("op", ["layer_norm_bwd", "linear_bwd", "glu_bwd"])
def test_workspace_sizes(op):
    cls, good = GOOD[op]
    size = getattr(sa.lib(), f"structadmm_{op}_workspace")
    d = cls(**good)
    need = size(ctypes.byref(d))
    assert need > 0
    d.ws, d.ws_bytes = FAKE * 32, need - 1
    assert getattr(sa.lib(), f"structadmm_{op}")(ctypes.byref(d), None) == -3
    bad = cls(**{**good, "type": 7})
    assert size(ctypes.byref(bad)) == 0 and size(None) == 0


def test_empty_products_need_no_pointers():
    """Zero rows: accepted with NULL matrices, and nothing to launch."""
    d = sa.LinearDesc(M=0, N=16, K=8, type=sa.BF16, out_type=sa.BF16, act=0, W=FAKE, ldx=8, ldw=8, ldy=16)
    assert sa.lib().structadmm_linear_fwd(ctypes.byref(d), None) == 0
    d = sa.LayerNormDesc(rows=0, cols=8, type=sa.F32, eps=1e-5, ldx=8, ldy=8)
    assert sa.lib().structadmm_layer_norm_fwd(ctypes.byref(d), None) == 0


def test_binding_refuses_what_is_no_gpu_matrix():
    import torch
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(sa.StructAdmmError, match="GPU memory"):
        sa.linear_fwd(x, x)
    with pytest.raises(sa.StructAdmmError, match="GPU memory"):
        sa.layer_norm_fwd(x)
    with pytest.raises(sa.StructAdmmError, match="GPU memory"):
        sa.glu_fwd(x, x, x)


def test_binding_checks_matrices():
    import torch
    dev = torch.device("cpu")
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    assert sa._matrix(x, 4, 8, sa.BF16, dev, "x") == 8
    assert sa._matrix(x[:, :5], 4, 5, sa.BF16, dev, "x") == 8
    assert sa._matrix(x.view(torch.uint16), 4, 8, sa.BF16, dev, "x") == 8
    assert sa._matrix(torch.zeros(1, 8).expand(1, 8), 1, 8, sa.F32, dev, "x") == 8
    for bad, rows, cols, code in [(x.t(), 8, 4, sa.BF16), (x, 4, 7, sa.BF16), (x, 4, 8, sa.F16), (x[0], 4, 8, sa.BF16),
                                  (x.double(), 4, 8, sa.BF16)]:
        with pytest.raises(sa.StructAdmmError):
            sa._matrix(bad, rows, cols, code, dev, "x")
    v = torch.zeros(8)
    assert sa._vector(v, 8, dev, "v") == v.data_ptr() and sa._vector(None, 8, dev, "v") is None
    for bad in (v[:7], v.double(), torch.zeros(16)[::2], v.view(2, 4)):
        with pytest.raises(sa.StructAdmmError):
            sa._vector(bad, 8, dev, "v")


def test_compacted_matrix_is_a_view():
    import torch
    sizes = sa.CompactSizes()
    sizes.groups, sizes.M[0], sizes.K[0], sizes.ldk[0], sizes.wc_offset[0] = 1, 3, 70, 128, 0
    wc = torch.arange(4 * 128, dtype=torch.int16).view(torch.uint16)
    m = sa.compacted_matrix(wc, sizes)
    assert m.shape == (3, 70) and m.stride() == (128, 1) and m.dtype == torch.bfloat16
    assert m.data_ptr() == wc.data_ptr()
    with pytest.raises(sa.StructAdmmError):
        sa.compacted_matrix(wc, sizes, 1)


def test_every_declared_operator_is_documented():
    """Each entry point of the header has its line in the binding's overview."""
    text = open(os.path.join(ROOT, "include", "structadmm.h")).read()
    for op in GOOD:
        assert re.search(rf"int structadmm_{op}\(", text) and f"  {op}(" in sa.__doc__, op
