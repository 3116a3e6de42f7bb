"""Which stream's memory the binding's own buffers are, in calls on a stream that is not the current one
(CPU only: a torch that records allocations, a library that launches nothing)."""

import contextlib
import os
import types

import pytest

from paper_2507_16697_amd import ringx

needs_lib = pytest.mark.skipif(not os.path.exists(ringx.LIB_PATH), reason="libringx.so not built")
HERE, THERE = 100, 200      # handles of the current stream and of the calls'
DEVICE = types.SimpleNamespace(index=0)


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class ExternalStream(Stream):
    def __init__(self, handle, device=None):
        super().__init__(handle)


class Torch:
    """The part of torch that the binding uses, on tensors without memory."""
    bfloat16, float32, float64, int32, int64, uint8, uint64 = "bf16 f32 f64 i32 i64 u8 u64".split()

    def __init__(self):
        self.made, self.now, self.calls = [], HERE, []
        torch = self

        class Tensor:
            is_cuda, device = True, DEVICE

            def __init__(self, shape, dtype):
                self.shape = (shape,) if isinstance(shape, int) else tuple(shape)
                self.dtype, self.pool, self.fills, self.users = dtype, torch.now, [], []

            def is_contiguous(self):
                return True

            def dim(self):
                return len(self.shape)

            def stride(self):
                st = [1]
                for n in self.shape[:0:-1]:
                    st.insert(0, st[0] * n)
                return tuple(st)

            def numel(self):
                n = 1
                for x in self.shape:
                    n *= x
                return n

            def element_size(self):
                return {"u8": 1, "bf16": 2}.get(self.dtype, 4)

            def data_ptr(self):
                return 0x10_0000 + 64 * id(self) % (1 << 40)

            def new_empty(self, shape, dtype):
                return torch.empty(shape, dtype=dtype)

            def zero_(self):
                self.fills.append(torch.now)
                return self

            def record_stream(self, s):
                self.users.append(s.cuda_stream)

        @contextlib.contextmanager
        def stream(s):
            old, torch.now = torch.now, s.cuda_stream
            yield
            torch.now = old

        self.Tensor = Tensor
        self.cuda = types.SimpleNamespace(
            Stream=Stream, ExternalStream=ExternalStream, stream=stream, current_device=lambda: 0,
            current_stream=lambda device=None: Stream(torch.now))

    def empty(self, shape, dtype, device=None):
        t = self.Tensor(shape, dtype)
        self.made.append(t)
        return t

    def empty_like(self, t):
        return self.empty(t.shape, t.dtype)

    def zeros(self, shape, dtype, device=None):
        return self.empty(shape, dtype).zero_()


@pytest.fixture
def torch(monkeypatch):
    t = Torch()
    real = ringx.lib()

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(real, name)
            return lambda *a: t.calls.append((name, a[-1])) or 0

    monkeypatch.setattr(ringx, "_T", t)
    monkeypatch.setattr(ringx, "_raw_stream", lambda index: t.now)
    monkeypatch.setattr(ringx, "lib", lambda: Lib())
    return t


def operands(torch, B=1, H=2, Nq=4096, Nk=4096, d=128):
    T, b, f = torch.Tensor, torch.bfloat16, torch.float32
    q, k = T((B, H, Nq, d), b), T((B, H, Nk, d), b)
    return types.SimpleNamespace(q=q, k=k, v=T(k.shape, b), out=T(q.shape, b), do=T(q.shape, b),
                                 lse=T((B, H, Nq), f), delta=T((2, B, H, Nq), f), rng=T((2,), torch.int64),
                                 dq=T(q.shape, f), dk=T(k.shape, f), dv=T(k.shape, f),
                                 qkv=T((B, Nq, 3 * H * d), b), freqs=T((d // 2,), torch.float64),
                                 w=T((d,), f), d=d, H=H)


WITH_WORKSPACE = {
    "bwd": lambda o, **kw: ringx.ringx_attn_bwd(o.q, o.k, o.v, o.out, o.do, o.lse, 4, **kw),
    "bwd_gqa": lambda o, **kw: ringx.ringx_attn_bwd_gqa(o.q, o.k, o.v, o.out, o.do, o.lse, 4, **kw),
    "bwd_ds": lambda o, **kw: ringx.ringx_attn_bwd_ds(o.q, o.k, o.v, o.out, o.do, o.lse, 4, **kw),
    "fwd_drop": lambda o, **kw: ringx.ringx_attn_fwd_drop(o.q, o.k, o.v, 0.1, o.rng, **kw),
    "bwd_drop": lambda o, **kw: ringx.ringx_attn_bwd_drop(o.q, o.k, o.v, o.out, o.do, o.lse, 0.1, o.rng,
                                                          **kw),
    "rope_bwd": lambda o, **kw: ringx.ringx_qkv_norm_rope_bwd(o.qkv, o.dq, o.dk, o.dv, o.freqs, (o.d,),
                                                              q_weight=o.w, **kw),
}


@needs_lib
@pytest.mark.parametrize("name", sorted(WITH_WORKSPACE))
@pytest.mark.parametrize("stream", [None, HERE, THERE, "object", "external"])
def test_hidden_workspaces_are_the_launch_streams(torch, name, stream):
    o = operands(torch)
    given = {"object": Stream(THERE), "external": types.SimpleNamespace(cuda_stream=THERE)}.get(stream, stream)
    WITH_WORKSPACE[name](o, stream=given)
    (_, launched), = torch.calls
    hidden = [t for t in torch.made if t.dtype == torch.uint8]
    assert launched == (HERE if stream in (None, HERE) else THERE)
    assert len(hidden) == 1 and hidden[0].pool == launched and torch.now == HERE


ALL = dict(WITH_WORKSPACE, **{
    "fwd": lambda o, **kw: ringx.ringx_attn_fwd(o.q, o.k, o.v, 4, **kw),
    "fwd_partials": lambda o, **kw: ringx.ringx_attn_fwd_partials(o.q, o.k, o.v, 4, **kw),
    "merge": lambda o, **kw: ringx.ringx_lse_merge(o.parts, o.part_lse, **kw),
    "pre": lambda o, **kw: ringx.ringx_bwd_preprocess(o.out, o.do, o.lse, **kw),
    "pre_drop": lambda o, **kw: ringx.ringx_bwd_preprocess_drop(o.out, o.do, o.lse, 0.1, **kw),
    "dkdv": lambda o, **kw: ringx.ringx_attn_bwd_dkdv(o.q, o.k, o.v, o.do, o.lse, o.delta, 4, **kw),
    "dq": lambda o, **kw: ringx.ringx_attn_bwd_dq(o.q, o.k, o.v, o.do, o.lse, o.delta, 4, **kw),
    "fwd_gqa": lambda o, **kw: ringx.ringx_attn_fwd_gqa(o.q, o.k, o.v, 4, **kw),
    "dkdv_ds": lambda o, **kw: ringx.ringx_attn_bwd_dkdv_ds(o.q, o.k, o.v, o.do, o.lse, o.delta, 4, o.ds, 0, 1,
                                                            **kw),
    "dq_ds": lambda o, **kw: ringx.ringx_attn_bwd_dq_ds(o.ds, o.k, o.q.shape, 4, 0, 1, **kw),
    "rope": lambda o, **kw: ringx.ringx_qkv_norm_rope(o.qkv, o.H, o.H, o.freqs, (o.d,), **kw),
    "tokenize": lambda o, **kw: ringx.ringx_tt_tokenize(o.field, 2, 1, (0, 0, 0), 4, **kw),
    "bwd +=": lambda o, **kw: ringx.ringx_attn_bwd(o.q, o.k, o.v, o.out, o.do, o.lse, 4, accumulate_dkv=True,
                                                   **kw),
    "bwd_drop +=": lambda o, **kw: ringx.ringx_attn_bwd_drop(o.q, o.k, o.v, o.out, o.do, o.lse, 0.1, o.rng,
                                                             accumulate_dkv=True, **kw),
})


@needs_lib
@pytest.mark.parametrize("name", sorted(ALL))
@pytest.mark.parametrize("stream", [None, HERE, THERE, "object"])
def test_buffers_handed_out_are_the_launch_streams(torch, name, stream):
    """Outputs that the caller does not give, and the zeros that gradients are added to."""
    o = operands(torch)
    o.parts, o.part_lse = torch.Tensor((4, 1, 2, 8, 64), torch.float32), torch.Tensor((4, 1, 2, 8), torch.float32)
    o.field, o.ds = torch.Tensor((1, 16, 16, 16), torch.float32), torch.Tensor((1 << 20,), torch.uint8)
    res = ALL[name](o, stream=Stream(THERE) if stream == "object" else stream)
    res = [t for t in (res if isinstance(res, tuple) else (res,)) if t is not None]
    (_, launched), = torch.calls
    assert launched == (HERE if stream in (None, HERE) else THERE)
    assert res and all(any(t is m for m in torch.made) for t in res) and torch.now == HERE
    for t in torch.made:
        assert t.pool == launched and all(f == launched for f in t.fills)
    for t in res:     # the caller's stream goes on to use them
        assert t.users == ([] if launched == HERE else [HERE])
    assert sum(len(t.fills) for t in torch.made) == (2 if "+=" in name or name == "dkdv_ds" else 0)
