"""CPU checks of the choice of exact products in the 8-bit products' C ABI and binding."""
import ctypes

import pytest

import paper_1807_11091_amd as sa
from test_abi_nn8 import FAKE, ask, good


@pytest.mark.parametrize("op", ["linear8_fwd", "glu8_fwd"])
@pytest.mark.parametrize("value", [-1, 2, 1 << 30])
def test_refuses_what_is_neither_0_nor_1(op, value):
    d = good(op)
    d.exact = value
    assert getattr(sa.lib(), f"structadmm_{op}")(ctypes.byref(d), None) == -1
    assert "exact" in sa.lib().structadmm_last_error().decode()
    assert ask(op[:-4], d) == 0


@pytest.mark.parametrize("op", ["linear8_fwd", "glu8_fwd"])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 9830), (16, 9830, 4096), (64, 640, 2000), (300, 2458, 1024), (130, 130, 16000)])
def test_workspace_of_exact_products(op, M, N, K):
    """Exact products go by the plan of a call with a binary32 or 8-bit result, and a query
    before the outputs covers them."""
    up = lambda n: (n + 127) // 128 * 128

    def desc(exact, y=FAKE, out_type=sa.BF16):
        x, w = sa.Matrix8Arg(FAKE, up(K), FAKE, 1, M), sa.Matrix8Arg(FAKE, up(K), FAKE, 1, up(N) // 128)
        none = sa.Matrix8Arg(None, up(N), None, 1, M)
        if op == "glu8_fwd":
            return sa.Glu8Desc(M=M, N=N, K=K, type=sa.BF16, act=0, X=x, Wg=w, Wu=w, ldh=N, ldgu=N, H=y, Q=none, exact=exact)
        return sa.Linear8Desc(M=M, N=N, K=K, type=sa.BF16, out_type=out_type, act=0, X=x, W=w, ldy=N, Y=y, Q=none, exact=exact)
    name = op[:-4]
    assert ask(name, desc(1)) <= ask(name, desc(1, None))
    assert ask(name, desc(0)) <= ask(name, desc(0, None))
    if op == "linear8_fwd":
        assert ask(name, desc(1)) == ask(name, desc(0, out_type=sa.F32))


@pytest.mark.parametrize("name", ["linear8_fwd", "glu8_fwd"])
def test_binding_passes_the_choice_on(name, monkeypatch):
    import torch
    seen = []
    monkeypatch.setattr(sa, "_run", lambda d, *a: seen.append(d.exact))
    monkeypatch.setattr(sa, "_codes_of", lambda m, what: m.codes.shape)
    dev = torch.device("cpu")
    X, W = sa.matrix8(4, 200, device=dev), sa.matrix8(300, 200, 128, device=dev)
    monkeypatch.setattr(sa, "_new", lambda stream, like, *shape: torch.empty(shape[:2], dtype=torch.bfloat16))
    monkeypatch.setattr(sa, "_optional", lambda t, *a: (None if t is None else 16, 300))
    monkeypatch.setattr(sa, "_type_code", lambda t, what: sa.BF16)
    call = (lambda **kw: sa.linear8_fwd(X, W, **kw)) if name == "linear8_fwd" else (lambda **kw: sa.glu8_fwd(X, W, W, out="h", **kw))
    call()
    call(exact=True)
    assert seen == [0, 1]
