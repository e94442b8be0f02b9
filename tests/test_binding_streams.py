"""The binding's own allocations for a call on another stream: memory of that
stream's pool, and the current stream marked as a user.  On the CPU, with stand-ins
for torch's streams, its allocator and the library; one GPU test at the end."""
import contextlib

import pytest

import paper_1807_11091_amd as sa


class Stand:
    """As much of a GPU tensor as the binding reads."""

    def __init__(self, shape, dtype):
        import torch
        self.shape = torch.Size((shape,) if isinstance(shape, int) else shape)
        self.dtype, self.device, self.is_cuda, self.users = dtype, torch.device("cuda", 0), True, []

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        import torch
        s = torch.empty(self.shape, device="meta").stride()
        return s if i is None else s[i]

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return 1

    def data_ptr(self):
        return id(self) // 256 * 256

    def is_contiguous(self):
        return True

    def record_stream(self, stream):
        self.users.append(stream)

    def __getitem__(self, at):
        import torch
        return Stand(torch.empty(self.shape, device="meta")[at].shape, self.dtype)


class Library:
    """Every workspace takes 512 bytes, every call succeeds."""

    def __getattr__(self, name):
        return (lambda *a: 512) if name.endswith("_workspace") else (lambda *a: 0)


class Stream:
    cuda_stream = 77


@pytest.fixture
def pools(monkeypatch):
    """The allocations of a call: (the stream whose pool they came from, tensor)."""
    import torch
    made, now = [], ["current"]
    real = torch.empty

    def empty(shape, dtype=None, device=None):
        if str(device) == "meta":
            return real(shape, device=device)
        made.append((now[-1], Stand(shape, dtype)))
        return made[-1][1]

    @contextlib.contextmanager
    def stream(s):
        now.append(s)
        yield
        now.pop()

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: ("handle", handle))
    monkeypatch.setattr(sa, "_raw_stream", lambda device: 5)
    monkeypatch.setattr(sa, "lib", lambda: Library())
    return made


def calls():
    import torch
    bf, f32, u16 = torch.bfloat16, torch.float32, torch.uint16
    M, N, K = 6, 10, 8
    X, Y, W, V = Stand((M, K), bf), Stand((M, N), bf), Stand((N, K), bf), Stand((N, K), bf)
    m, Z4 = Stand(M, f32), Stand((4, 4, 3, 3), f32)
    sizes = sa.CompactSizes()
    sizes.groups, sizes.M[0] = 1, 4
    Xp, idx = Stand((1, 8, 8, 4), u16), Stand(9, torch.int32)
    return {
        "layer_norm_fwd": lambda s: sa.layer_norm_fwd(X, stream=s),
        "layer_norm_bwd": lambda s: sa.layer_norm_bwd(X, X, m, m, stream=s),
        "linear_fwd": lambda s: sa.linear_fwd(X, W, stream=s),
        "linear_bwd": lambda s: sa.linear_bwd(Y, X, W, grads="xwb", stream=s),
        "glu_fwd": lambda s: sa.glu_fwd(X, W, V, stream=s),
        "glu_bwd": lambda s: sa.glu_bwd(Y, X, W, V, Y, Y, grads="xwb", stream=s),
        "compact": lambda s: sa.compact(Z4, stream=s),
        "compact_many": lambda s: sa.compact_many([dict(Z=Z4), dict(Z=Z4)], stream=s),
        "pack_nhwc": lambda s: sa.pack_nhwc(Stand((1, 4, 8, 8), f32), stream=s),
        "conv_fwd": lambda s: sa.conv_fwd(Xp, idx, idx, idx, sizes, 3, 3, 1, 1, stream=s),
        "csr": lambda s: sa.csr(Z4, idx, stream=s),
        "conv_sparse_fwd": lambda s: sa.conv_sparse_fwd(Xp, idx, idx, idx, (4, 4, 3, 3), 1, 1, 1, 9, stream=s),
    }


@pytest.mark.parametrize("name", list(calls()))
def test_memory_comes_from_the_streams_pool(pools, name):
    s = Stream()
    calls()[name](s)
    assert pools
    for pool, t in pools:
        assert pool is s, (name, t.shape)
        assert "current" in t.users, (name, t.shape)


@pytest.mark.parametrize("name", list(calls()))
def test_memory_for_a_raw_handle(pools, name):
    calls()[name](88)
    assert pools
    for pool, t in pools:
        assert pool == ("handle", 88) and "current" in t.users, (name, t.shape)


@pytest.mark.parametrize("handle", [None, 5])
@pytest.mark.parametrize("name", list(calls()))
def test_memory_on_the_current_stream(pools, name, handle):
    calls()[name](handle)
    assert pools and all(pool == "current" and not t.users for pool, t in pools)


@pytest.mark.parametrize("name", ["layer_norm_bwd", "linear_fwd", "linear_bwd", "glu_fwd", "glu_bwd"])
def test_workspaces_that_are_refused(pools, name):
    """A workspace in host memory, or a view whose elements lie apart, is not handed to
    the kernels."""
    import torch
    bf, f32 = torch.bfloat16, torch.float32
    X, Y, W, V, m = Stand((6, 8), bf), Stand((6, 10), bf), Stand((10, 8), bf), Stand((10, 8), bf), Stand(6, f32)
    args = {"layer_norm_bwd": (X, X, m, m), "linear_fwd": (X, W), "linear_bwd": (Y, X, W), "glu_fwd": (X, W, V),
            "glu_bwd": (Y, X, W, V, Y, Y)}[name]
    call = getattr(sa, name)
    call(*args, ws=Stand(4096, torch.uint8))
    with pytest.raises(sa.StructAdmmError, match="ws must be contiguous and on cuda:0"):
        call(*args, ws=torch.zeros(4096, dtype=torch.uint8))
    apart = Stand(4096, torch.uint8)
    apart.is_contiguous = lambda: False
    with pytest.raises(sa.StructAdmmError, match="contiguous"):
        call(*args, ws=apart)


@pytest.mark.gpu
@pytest.mark.parametrize("raw", [False, True])
def test_a_busy_block_is_not_taken(raw):
    """A block that was dropped while the current stream still works on it is not
    given to a call on another stream, whose result is right all the same."""
    import torch
    M, N, K = 512, 1024, 1024
    g = torch.Generator(device="cuda").manual_seed(1)
    X, W = (torch.randn(n, K, generator=g, device="cuda").bfloat16() for n in (M, N))
    want = sa.linear_fwd(X, W)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(4):
        busy = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        at = busy.data_ptr()
        for _ in range(50):
            busy.fill_(7.0)
        keep = busy.float()
        del busy
        got = sa.linear_fwd(X, W, stream=side.cuda_stream if raw else side)
        assert got.data_ptr() != at
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want) and (keep == 7.0).all()
        del got
    with torch.cuda.stream(side):
        got = sa.linear_fwd(X, W, stream=torch.cuda.default_stream().cuda_stream)  # the null stream's handle
        side.wait_stream(torch.cuda.default_stream())
        assert torch.equal(got, want)
