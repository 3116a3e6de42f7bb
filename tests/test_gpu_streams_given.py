"""Calls on a stream that is not the current one (stream=...): what the current stream allocates while they
run is not theirs."""

import pytest
import torch

from paper_2507_16697_amd import inputs, ringx

from parity_util import to_device

pytestmark = pytest.mark.gpu

B, H, HKV, N, D = 1, 2, 2, 4096, 128      # a size whose dropout forward and backward both take parts


def operands():
    a = inputs.make_iid(B, H, N, N, D, seed=5, std=0.7, store="bf16")
    t = {n: to_device(a[n], "bf16") for n in ("q", "k", "v", "do")}
    t["rng"] = torch.tensor([3, 4], device="cuda")
    t["out"], t["lse"] = ringx.ringx_attn_fwd_drop(t["q"], t["k"], t["v"], 0.1, t["rng"])
    g = torch.Generator().manual_seed(6)
    t["qkv"] = torch.randn((B, N, 3 * H * D), generator=g).to("cuda", torch.bfloat16)
    t["grads"] = [torch.randn((B, H, N, D), generator=g).cuda() for _ in range(3)]
    t["freqs"] = 10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    t["w"] = torch.ones(D, device="cuda")
    return t


CALLS = {
    "bwd": lambda t, **kw: ringx.ringx_attn_bwd(t["q"], t["k"], t["v"], t["out"], t["do"], t["lse"], 4, **kw),
    "bwd_gqa": lambda t, **kw: ringx.ringx_attn_bwd_gqa(t["q"], t["k"], t["v"], t["out"], t["do"], t["lse"], 4,
                                                        **kw),
    "bwd_ds": lambda t, **kw: ringx.ringx_attn_bwd_ds(t["q"], t["k"], t["v"], t["out"], t["do"], t["lse"], 4,
                                                      **kw),
    "fwd_drop": lambda t, **kw: ringx.ringx_attn_fwd_drop(t["q"], t["k"], t["v"], 0.1, t["rng"], **kw),
    "bwd_drop": lambda t, **kw: ringx.ringx_attn_bwd_drop(t["q"], t["k"], t["v"], t["out"], t["do"], t["lse"],
                                                          0.1, t["rng"], **kw),
    "rope_bwd": lambda t, **kw: ringx.ringx_qkv_norm_rope_bwd(t["qkv"], *t["grads"], t["freqs"], (D,),
                                                              q_weight=t["w"], k_weight=t["w"], **kw),
}
BYTES = {
    "bwd": lambda: ringx.ringx_bwd_workspace_bytes(B, H, N, N, D, 4, ringx.RINGX_BF16),
    "bwd_gqa": lambda: ringx.ringx_bwd_workspace_bytes(B, H, N, N, D, 4, ringx.RINGX_BF16),
    "bwd_ds": lambda: ringx.ringx_bwd_ds_workspace_bytes(B, H, HKV, N, N, D, 4, 2),
    "fwd_drop": lambda: ringx.ringx_fwd_drop_workspace_bytes(B, H, HKV, N, N, D, ringx.RINGX_BF16),
    "bwd_drop": lambda: ringx.ringx_bwd_drop_workspace_bytes(B, H, HKV, N, N, D, ringx.RINGX_BF16),
    "rope_bwd": lambda: ringx.ringx_qkv_norm_rope_bwd_workspace_bytes(B, N, H, HKV, D, ringx.RINGX_BF16),
}


def on_a_held_up_stream(side, call):
    """call() with `side` busy for some milliseconds, so that what it launches there runs later."""
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(5_000_000)
    return call()


def buffers_like(sizes):
    """What the current stream allocates next: buffers of these sizes, several of each, all ones."""
    return [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]


@pytest.mark.parametrize("form", ["stream", "handle", "default"])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_workspaces_of_calls_on_another_stream(name, form):
    print(f"{name} on a {form}", flush=True)
    t = operands()
    want = CALLS[name](t)
    torch.cuda.synchronize()
    here = torch.cuda.current_stream()
    other = torch.cuda.Stream()
    side = here if form == "default" else other          # the default stream, while another is current
    now = other if form == "default" else here
    given = {"stream": side, "handle": side.cuda_stream, "default": 0}[form]
    with torch.cuda.stream(now):
        for _ in range(3):
            got = on_a_held_up_stream(side, lambda: CALLS[name](t, stream=given))
            junk = buffers_like([BYTES[name]()])
            torch.cuda.synchronize()
            assert all(bool((x == 255).all()) for x in junk)
            assert all(torch.equal(a, b) for a, b in zip(want, got))
            del junk


CALLS_HANDING_OUT = dict(CALLS, **{
    "fwd": lambda t, **kw: ringx.ringx_attn_fwd(t["q"], t["k"], t["v"], 4, **kw),
    "fwd_partials": lambda t, **kw: ringx.ringx_attn_fwd_partials(t["q"], t["k"], t["v"], 4, **kw),
    "rope": lambda t, **kw: ringx.ringx_qkv_norm_rope(t["qkv"], H, H, t["freqs"], (D,), **kw),
    "bwd +=": lambda t, **kw: ringx.ringx_attn_bwd(t["q"], t["k"], t["v"], t["out"], t["do"], t["lse"], 4,
                                                   accumulate_dkv=True, **kw),
    "bwd_drop +=": lambda t, **kw: ringx.ringx_attn_bwd_drop(t["q"], t["k"], t["v"], t["out"], t["do"],
                                                             t["lse"], 0.1, t["rng"], accumulate_dkv=True,
                                                             **kw),
})


@pytest.mark.parametrize("name", sorted(CALLS_HANDING_OUT))
def test_outputs_of_calls_on_another_stream(name):
    """Outputs may be dropped before they are written; gradients are added to zeros, not to what the fill
    has still to clear."""
    print(name, flush=True)
    call = CALLS_HANDING_OUT[name]
    t = operands()
    want = call(t)
    sizes = [x.numel() * x.element_size() for x in want]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for keep in range(len(want)):
        got = on_a_held_up_stream(side, lambda: call(t, stream=side)[keep])
        junk = buffers_like(n for i, n in enumerate(sizes) if i != keep)
        torch.cuda.synchronize()
        assert all(bool((x == 255).all()) for x in junk) and torch.equal(got, want[keep])
        del junk


def test_a_call_on_another_stream_is_captured():
    """The launch stream forked from a capturing one: its buffers belong to the graph."""
    t = operands()
    want = CALLS["fwd_drop"](t) + CALLS["bwd_drop"](t)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    main.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(main), torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        got = CALLS["fwd_drop"](t, stream=side) + CALLS["bwd_drop"](t, stream=side)
        main.wait_stream(side)
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
        junk = buffers_like([BYTES["fwd_drop"](), BYTES["bwd_drop"]()])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        assert all(bool((x == 255).all()) for x in junk)
        for x in got:
            x.zero_()
