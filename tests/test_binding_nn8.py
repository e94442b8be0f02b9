"""The binding of the 8-bit operators on the CPU, with stand-ins for torch's streams, its
allocator and the library: memory from the right stream's pool, refused workspaces, types."""
import pytest

import paper_1807_11091_amd as sa
from test_binding_streams import Library, Stand, Stream, pools  # noqa: F401  (pools is a fixture)


@pytest.fixture(autouse=True)
def matrices(monkeypatch):
    import torch
    monkeypatch.setattr(Stand, "view", lambda self, dtype: Stand(self.shape, dtype), raising=False)

    def turned(self):
        s = Stand(tuple(reversed(self.shape)), self.dtype)
        s.stride = lambda i=None: (1, self.shape[1])
        return s
    monkeypatch.setattr(Stand, "t", turned, raising=False)
    real = Stand.__getitem__

    def part(self, at):  # a view keeps its pitch
        s = real(self, at)
        if isinstance(at, tuple) and self.dtype == torch.float8_e4m3fn:
            s.stride = lambda i=None: (self.shape[1], 1)
        return s
    monkeypatch.setattr(Stand, "__getitem__", part)


def eight(rows, cols, block=1):
    import torch
    up = lambda n: (n + 127) // 128
    codes = Stand((rows, up(cols) * 128), torch.float8_e4m3fn)[:, :cols]
    return sa.Matrix8(codes, Stand((up(cols), rows if block == 1 else up(rows)), torch.float32).t())


def calls():
    import torch
    bf, f32 = torch.bfloat16, torch.float32
    M, N, K = 6, 300, 200
    X, W, V = eight(M, K), eight(N, K, 128), eight(N, K, 128)
    x, m = Stand((M, K), bf), Stand(M, f32)
    return {
        "rms_norm_fwd": lambda s: sa.rms_norm_fwd(x, R=x, out="ysrq", stream=s),
        "rms_norm_bwd": lambda s: sa.rms_norm_bwd(x, x, m, stream=s),
        "quantize8": lambda s: sa.quantize8(x, out="qt", stream=s),
        "linear8_fwd": lambda s: sa.linear8_fwd(X, W, out="yq", stream=s),
        "glu8_fwd": lambda s: sa.glu8_fwd(X, W, V, out="hq", stream=s),
        "matrix8": lambda s: sa.matrix8(M, N, device=x.device, stream=s),
    }


@pytest.mark.parametrize("name", ["rms_norm_fwd", "rms_norm_bwd", "quantize8", "linear8_fwd", "glu8_fwd", "matrix8"])
def test_memory_comes_from_the_streams_pool(pools, name):  # noqa: F811
    s = Stream()
    calls()[name](s)
    assert pools
    for pool, t in pools:
        assert pool is s and "current" in t.users, (name, t.shape)
    pools.clear()
    calls()[name](88)
    for pool, t in pools:
        assert pool == ("handle", 88) and "current" in t.users, (name, t.shape)
    pools.clear()
    calls()[name](None)
    assert pools and all(pool == "current" and not t.users for pool, t in pools)


@pytest.mark.parametrize("name", ["rms_norm_bwd", "linear8_fwd", "glu8_fwd"])
def test_workspaces_that_are_refused(pools, name):  # noqa: F811
    import torch
    x, m = Stand((6, 200), torch.bfloat16), Stand(6, torch.float32)
    X, W = eight(6, 200), eight(300, 200, 128)
    args = {"rms_norm_bwd": (x, x, m), "linear8_fwd": (X, W), "glu8_fwd": (X, W, W)}[name]
    getattr(sa, name)(*args, ws=Stand(4096, torch.uint8))
    with pytest.raises(sa.StructAdmmError, match="ws must be contiguous and on cuda:0"):
        getattr(sa, name)(*args, ws=torch.zeros(4096, dtype=torch.uint8))


def test_types_of_results(pools):  # noqa: F811
    import torch
    X, W = eight(6, 200), eight(300, 200, 128)
    bf, half, f32 = torch.bfloat16, torch.float16, torch.float32
    new = lambda t: Stand((6, 300), t)
    assert sa.linear8_fwd(X, W)[0].dtype == bf
    assert sa.linear8_fwd(X, W, R=new(half))[0].dtype == half
    assert sa.linear8_fwd(X, W, Z=new(half))[0].dtype == half
    assert sa.linear8_fwd(X, W, out_dtype=f32)[0].dtype == f32
    assert sa.linear8_fwd(X, W, Z=new(bf), out_dtype=f32)[0].dtype == f32
    assert sa.linear8_fwd(X, W, out="q")[0] is None
    assert sa.glu8_fwd(X, W, W, out="h")[0].dtype == bf
    assert sa.glu8_fwd(X, W, W, G=new(half), U=new(half), out="hq")[0].dtype == half
    with pytest.raises(sa.StructAdmmError, match="type"):
        sa.linear8_fwd(X, W, Y=new(bf), R=new(f32))
    with pytest.raises(sa.StructAdmmError, match="both G and U"):
        sa.glu8_fwd(X, W, W, G=new(bf))
    with pytest.raises(sa.StructAdmmError, match="scales"):
        sa.linear8_fwd(X, eight(300, 200))
    with pytest.raises(sa.StructAdmmError, match="block_rows"):
        sa.quantize8(Stand((6, 200), bf), 64)
    with pytest.raises(sa.StructAdmmError, match="rstd"):
        sa.rms_norm_bwd(new(bf), new(bf), None)
