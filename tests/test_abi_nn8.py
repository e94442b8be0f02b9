"""CPU checks of the 8-bit feed-forward operators' C ABI and binding: struct layouts,
refusals on the host (nothing is enqueued on these paths), workspace sizes."""
import ctypes
import os
import re
import subprocess

import pytest

import paper_1807_11091_amd as sa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # a 256-byte aligned non-null address; never dereferenced on these paths
STRUCTS = {"sa_matrix8": sa.Matrix8Arg, "sa_rms_norm_desc": sa.RmsNormDesc, "sa_rms_norm_bwd_desc": sa.RmsNormBwdDesc,
           "sa_quantize8_desc": sa.Quantize8Desc, "sa_linear8_desc": sa.Linear8Desc, "sa_glu8_desc": sa.Glu8Desc}


def test_struct_layouts_match_header(tmp_path):
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "structadmm.h"', "int main(void){"]
    for st, cls in STRUCTS.items():
        lines.append(f'printf("{st} sizeof %zu\\n", sizeof({st}));')
        lines += [f'printf("{st} {f} %zu\\n", offsetof({st}, {f}));' for f, _ in cls._fields_]
    lines += ['printf("const SA_BLOCK %d\\n", SA_BLOCK);', "return 0;}"]
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
    assert got[("const", "SA_BLOCK")] == sa.BLOCK


def eight(i, ld=16, row=1, col=4):
    return sa.Matrix8Arg(FAKE * i, ld, FAKE * (i + 1), row, col)


def addresses(*names, first=20):
    return {n: FAKE * (first + i) for i, n in enumerate(names)}


def good(op):
    if op == "rms_norm_fwd":
        return sa.RmsNormDesc(rows=4, cols=8, type=sa.BF16, eps=1e-5, ldx=8, ldr=8, lds=8, ldy=8, Q=eight(1),
                              **addresses("X", "R", "gamma", "S", "Y", "rstd"))
    if op == "rms_norm_bwd":
        return sa.RmsNormBwdDesc(rows=4, cols=8, type=sa.F16, lddy=8, lds=8, lddr=8, lddx=8,
                                 **addresses("dY", "S", "rstd", "gamma", "dR", "dX", "dgamma"))
    if op == "quantize8":
        return sa.Quantize8Desc(rows=4, cols=300, type=sa.F32, block_rows=1, ldx=300, Q=eight(1, 304, 1, 4),
                                QT=eight(3, 16, 1, 300), **addresses("X"))
    if op == "linear8_fwd":
        return sa.Linear8Desc(M=4, N=200, K=130, type=sa.BF16, out_type=sa.BF16, act=sa.ACT_SILU, X=eight(1, 144),
                              W=eight(3, 144, 1, 2), ldr=200, ldy=200, ldz=200, Q=eight(5, 208),
                              **addresses("bias", "R", "Y", "Z"))
    return sa.Glu8Desc(M=4, N=200, K=130, type=sa.F16, act=sa.ACT_SILU, X=eight(1, 144), Wg=eight(3, 144, 1, 2),
                       Wu=eight(5, 144, 1, 2), ldh=200, ldgu=200, Q=eight(7, 208), **addresses("bg", "bu", "H", "G", "U"))


OPS = ["rms_norm_fwd", "rms_norm_bwd", "quantize8", "linear8_fwd", "glu8_fwd"]
NONE = sa.Matrix8Arg(None, 304, None, 1, 1)
REFUSED = [
    ("rms_norm_fwd", dict(rows=-1), -1), ("rms_norm_fwd", dict(cols=0), -1), ("rms_norm_fwd", dict(type=3), -1),
    ("rms_norm_fwd", dict(X=None), -1), ("rms_norm_fwd", dict(eps=-1.0), -1), ("rms_norm_fwd", dict(eps=float("nan")), -1),
    ("rms_norm_fwd", dict(ldr=7), -1), ("rms_norm_fwd", dict(X=FAKE + 1), -2), ("rms_norm_fwd", dict(gamma=FAKE + 2), -2),
    ("rms_norm_fwd", dict(S=None, Y=None, Q=NONE, rstd=None), -1), ("rms_norm_fwd", dict(S=20 * FAKE, lds=9), -1),
    ("rms_norm_fwd", dict(S=21 * FAKE, lds=9), -1), ("rms_norm_fwd", dict(Y=23 * FAKE), -1),
    ("rms_norm_fwd", dict(Q=eight(1, 24)), -2), ("rms_norm_fwd", dict(Q=eight(1, 0)), -1),
    ("rms_norm_fwd", dict(Q=sa.Matrix8Arg(FAKE + 8, 16, 2 * FAKE, 1, 4)), -2),
    ("rms_norm_fwd", dict(Q=sa.Matrix8Arg(FAKE, 16, 2 * FAKE + 2, 1, 4)), -2),
    ("rms_norm_fwd", dict(Q=sa.Matrix8Arg(FAKE, 16, None, 1, 4)), -1), ("rms_norm_fwd", dict(Q=eight(1, 16, 0, 4)), -1),
    ("rms_norm_fwd", dict(Q=eight(1, 16, -1, 4)), -1), ("rms_norm_fwd", dict(Q=eight(20, 16)), -1),
    ("rms_norm_fwd", dict(Q=eight(22, 16)), -1), ("rms_norm_fwd", dict(Q=eight(1, 16, (1 << 21) + 1, 1)), -4),
    ("rms_norm_bwd", dict(rstd=None), -1), ("rms_norm_bwd", dict(dX=None, dgamma=None), -1),
    ("rms_norm_bwd", dict(dX=21 * FAKE), -1), ("rms_norm_bwd", dict(dY=None), -1), ("rms_norm_bwd", dict(lddr=7), -1),
    ("rms_norm_bwd", dict(type=9), -1), ("rms_norm_bwd", {}, -3),
    ("quantize8", dict(rows=-1), -1), ("quantize8", dict(rows=1 << 31), -1), ("quantize8", dict(cols=-1), -1),
    ("quantize8", dict(type=3), -1), ("quantize8", dict(block_rows=64), -1), ("quantize8", dict(X=None), -1),
    ("quantize8", dict(Q=NONE, QT=NONE), -1), ("quantize8", dict(Q=eight(1, 300)), -2),
    ("quantize8", dict(Q=eight(1, 288)), -1), ("quantize8", dict(Q=eight(1, 304, 1, 3)), -1),
    ("quantize8", dict(Q=eight(1, 304, 2, 1)), -1), ("quantize8", dict(QT=eight(3, 16, 0, 300)), -1),
    ("quantize8", dict(QT=eight(1, 16, 1, 300)), -1), ("quantize8", dict(Q=eight(20, 304)), -1),
    ("quantize8", dict(Q=eight(1, (1 << 21) + 16)), -4),
    ("quantize8", dict(rows=(1 << 21) + 1, Q=NONE, QT=eight(3, (1 << 21) + 16, 1, 300)), -4),
    ("linear8_fwd", dict(M=-1), -1), ("linear8_fwd", dict(type=sa.F32), -4), ("linear8_fwd", dict(type=9), -1),
    ("linear8_fwd", dict(out_type=sa.F16), -1), ("linear8_fwd", dict(act=6), -1), ("linear8_fwd", dict(X=NONE), -1),
    ("linear8_fwd", dict(W=NONE), -1), ("linear8_fwd", dict(Y=None, Q=NONE), -1), ("linear8_fwd", dict(X=eight(1, 136)), -2),
    ("linear8_fwd", dict(W=eight(3, 128)), -1), ("linear8_fwd", dict(X=eight(1, 144, -1)), -1),
    ("linear8_fwd", dict(X=eight(1, 144, 1, 1 << 31)), -4), ("linear8_fwd", dict(ldr=199), -1),
    ("linear8_fwd", dict(ldz=199), -1), ("linear8_fwd", dict(Y=FAKE), -1), ("linear8_fwd", dict(Y=2 * FAKE), -1),
    ("linear8_fwd", dict(Z=22 * FAKE), -1), ("linear8_fwd", dict(Y=21 * FAKE, ldy=201), -1),
    ("linear8_fwd", dict(Q=eight(22, 208)), -1), ("linear8_fwd", dict(Q=eight(3, 208)), -1),
    ("linear8_fwd", dict(Q=eight(21, 208)), -1), ("linear8_fwd", dict(Q=eight(5, 208, 1, 3)), -1),
    ("linear8_fwd", dict(K=(1 << 21) + 1), -4), ("linear8_fwd", dict(bias=FAKE * 20 + 1), -2),
    ("glu8_fwd", dict(G=None), -1), ("glu8_fwd", dict(Wu=NONE), -1), ("glu8_fwd", dict(Wu=eight(5, 160, 1, 2)), -1),
    ("glu8_fwd", dict(Wu=eight(5, 144, 2, 1)), -1), ("glu8_fwd", dict(H=None, Q=NONE), -1), ("glu8_fwd", dict(H=FAKE), -1),
    ("glu8_fwd", dict(U=23 * FAKE), -1), ("glu8_fwd", dict(ldgu=199), -1), ("glu8_fwd", dict(Q=eight(22, 208)), -1),
    ("glu8_fwd", dict(act=-1), -1),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refusals(i):
    op, kw, code = REFUSED[i]
    d = good(op)
    for k, v in kw.items():
        setattr(d, k, v)
    rc = getattr(sa.lib(), f"structadmm_{op}")(ctypes.byref(d), None)
    msg = sa.lib().structadmm_last_error().decode()
    assert rc == code, (op, kw, msg)
    assert op in msg


@pytest.mark.parametrize("op", OPS)
def test_null_descriptor(op):
    assert getattr(sa.lib(), f"structadmm_{op}")(None, None) == -1


def ask(name, d):
    return getattr(sa.lib(), f"structadmm_{name}_workspace")(ctypes.byref(d))


@pytest.mark.parametrize("op,name", [("linear8_fwd", "linear8"), ("glu8_fwd", "glu8"), ("rms_norm_bwd", "rms_norm_bwd")])
def test_workspace_sizes(op, name):
    """A call refuses one byte less than the query says; a query before the outputs
    covers every choice of them."""
    d = good(op)
    need = ask(name, d)
    if need:
        d.ws, d.ws_bytes = FAKE * 40, need - 1
        assert getattr(sa.lib(), f"structadmm_{op}")(ctypes.byref(d), None) == -3
    bad = good(op)
    bad.type = 7
    assert ask(name, bad) == 0 and getattr(sa.lib(), f"structadmm_{name}_workspace")(None) == 0


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 4096, 9830), (16, 9830, 4096), (64, 640, 2000), (300, 2458, 1024),
                                   (1000, 1024, 1229), (8192, 4096, 9830)])
def test_query_before_the_outputs(M, N, K):
    up = lambda n: (n + 127) // 128 * 128
    for gated in (False, True):
        def desc(y, q):
            x, w, o = sa.Matrix8Arg(FAKE, up(K), FAKE, 1, M), sa.Matrix8Arg(FAKE, up(K), FAKE, 1, up(N) // 128), \
                sa.Matrix8Arg(FAKE if q else None, up(N), FAKE, 1, M)
            if gated:
                return sa.Glu8Desc(M=M, N=N, K=K, type=sa.BF16, act=0, X=x, Wg=w, Wu=w, ldh=N, ldgu=N, H=y, Q=o)
            return sa.Linear8Desc(M=M, N=N, K=K, type=sa.BF16, out_type=sa.BF16, act=0, X=x, W=w, ldy=N, Y=y, Q=o)
        name = "glu8" if gated else "linear8"
        bare = ask(name, desc(None, False))
        for y, q in ((FAKE, False), (None, True), (FAKE, True)):
            assert ask(name, desc(y, q)) <= bare
            assert y is None or ask(name, desc(y, False)) <= ask(name, desc(FAKE, True))  # fewer outputs
        before = desc(None, False)  # nor do the operands have to be there
        before.X.codes = before.X.scales = None
        assert ask(name, before) == bare


def test_empty_calls_need_no_pointers():
    L = sa.lib()
    d = sa.Linear8Desc(M=0, N=16, K=8, type=sa.BF16, out_type=sa.BF16, X=NONE, W=eight(1), ldy=16, Q=NONE)
    assert L.structadmm_linear8_fwd(ctypes.byref(d), None) == 0
    d = sa.RmsNormDesc(rows=0, cols=8, type=sa.F32, eps=1e-5, ldx=8, Q=NONE)
    assert L.structadmm_rms_norm_fwd(ctypes.byref(d), None) == 0
    d = sa.Quantize8Desc(rows=0, cols=8, type=sa.F32, block_rows=128, ldx=8, Q=NONE, QT=NONE)
    assert L.structadmm_quantize8(ctypes.byref(d), None) == 0


def test_binding_refuses_what_is_no_gpu_matrix():
    import torch
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    m = sa.Matrix8(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1))
    for call in (lambda: sa.rms_norm_fwd(x), lambda: sa.quantize8(x), lambda: sa.linear8_fwd(m, m),
                 lambda: sa.glu8_fwd(m, m, m), lambda: sa.rms_norm_bwd(x, x, None), lambda: sa.linear8_fwd(x, m)):
        with pytest.raises(sa.StructAdmmError, match="GPU memory"):
            call()
    with pytest.raises(sa.StructAdmmError, match="block_rows"):
        sa.matrix8(4, 4, 64)


def test_binding_checks_8_bit_matrices():
    import torch
    dev = torch.device("cpu")
    m = sa.matrix8(5, 300, device=dev)
    assert m.codes.shape == (5, 300) and m.codes.stride() == (384, 1) and m.codes.dtype == torch.float8_e4m3fn
    assert m.scales.shape == (5, 3) and m.scales.stride() == (1, 5)
    a = sa._matrix8(m, 5, 300, 1, dev, "m")
    assert (a.codes, a.ld, a.scales, a.scale_row, a.scale_col) == (m.codes.data_ptr(), 384, m.scales.data_ptr(), 1, 5)
    w = sa.matrix8(300, 130, 128, device=dev)
    assert w.scales.shape == (3, 2) and sa._matrix8(w, 300, 130, 128, dev, "w").scale_col == 3
    assert sa._matrix8(sa.Matrix8(w.codes.view(torch.uint8), w.scales.contiguous()), 300, 130, 128, dev, "w").scale_row == 2
    one = sa.Matrix8(torch.zeros(300, dtype=torch.uint8).expand(1, 300), torch.zeros(1, 1).expand(1, 3))
    a = sa._matrix8(one, 1, 300, 1, dev, "one")  # a single row has no pitch; one scale for all its blocks
    assert a.ld == 304 and a.scale_col == 0
    none = sa._matrix8(None, 5, 300, 1, dev, "none")
    assert none.codes is None and none.ld == 304
    for bad in (sa.Matrix8(m.codes[:4], m.scales), sa.Matrix8(m.codes, m.scales[:, :2]), sa.Matrix8(m.codes, m.scales.double()),
                sa.Matrix8(m.codes.float(), m.scales), sa.Matrix8(m.codes.view(torch.uint8).t().contiguous().t(), m.scales),
                sa.Matrix8(m.codes, torch.zeros(1, 3))):
        with pytest.raises(sa.StructAdmmError):
            sa._matrix8(bad, 5, 300, 1, dev, "m")


def test_every_declared_operator_is_documented():
    text = open(os.path.join(ROOT, "include", "structadmm.h")).read()
    for op in OPS:
        assert re.search(rf"int structadmm_{op}\(", text) and f"  {op}(" in sa.__doc__, op
