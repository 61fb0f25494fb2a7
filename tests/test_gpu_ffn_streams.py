"""GPU: projections on streams that the calls are given, with workspaces of their own and without."""
import math

import pytest
import torch

import _projections as pj
from oracle import ffn as of
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu

M, N, K = 256, 1024, 16384
KINDS = (D.LINEAR_W4, D.GATED_LINEAR_BF16, D.GATED_LINEAR_W4)


class _Calls:
    """What projections are called with, one set of weights and outputs for each stream."""

    def __init__(self, count):
        dev = torch.device("cuda:0")
        gen = torch.Generator(device=dev)
        gen.manual_seed(4)
        normal = lambda *s: torch.empty(s, device=dev).normal_(generator=gen)  # noqa: E731
        self.w = [rt.Weights4.of(*pj.random_codes(gen, N, K, device=dev)) for _ in range(count + 1)]
        self.dense = [(normal(N, K) * 0.02).to(torch.bfloat16) for _ in range(count + 1)]
        self.x = [normal(M, K).to(torch.bfloat16) for _ in range(count)]
        self.out = [[torch.empty((M, N), dtype=torch.float32, device=dev) for _ in range(3)]
                    for _ in range(count)]

    def run(self, i, **how):
        rt.linear(self.x[i], self.w[i], self.out[i][0], **how)
        rt.gated_linear(self.x[i], self.dense[i], self.dense[i + 1], self.out[i][1], **how)
        rt.gated_linear(self.x[i], self.w[i], self.w[i + 1], self.out[i][2], "gelu", **how)

    def take(self):
        torch.cuda.synchronize()
        kept = [[t.clone() for t in ts] for ts in self.out]
        for ts in self.out:
            for t in ts:
                t.fill_(math.nan)
        torch.cuda.synchronize()
        return kept


def _workspace():
    sizes = [D.dlfp_projection_workspace(kind, M, N, K) for kind in KINDS]
    assert min(sizes) > 0
    room = torch.full((max(sizes),), 0xff, dtype=torch.uint8, device="cuda:0")
    torch.cuda.synchronize()
    return room


def test_a_stream_by_hand():
    """With a workspace what the current stream's calls give, bit for bit; without, K in one part."""
    calls, stream = _Calls(1), torch.cuda.Stream()
    calls.run(0)
    want = calls.take()[0]
    room = _workspace()
    for handle in (stream, stream.cuda_stream):
        calls.run(0, stream=handle, workspace=room)
        assert all(torch.equal(a, b) for a, b in zip(calls.take()[0], want))
    for kind in KINDS:
        assert D.dlfp_projection_form_of(kind, M, N, K, 0).splits == 1
    calls.run(0, stream=stream)
    whole = calls.take()[0]
    x = pj.f64(calls.x[0][:4])
    gate, up = (of.values(w.codes.cpu().numpy(), w.exps.cpu().numpy()) for w in calls.w)
    for got, expected in zip(whole, (pj.linear(x, gate, torch.float32),
                                     pj.gated(x, *map(pj.f64, calls.dense), "silu", torch.float32),
                                     pj.gated(x, gate, up, "gelu", torch.float32))):
        pj.check(got[:4], *expected)


def test_two_streams_by_hand_and_their_graphs():
    """Side by side, eager and as a graph of each, a workspace for each stream."""
    calls = _Calls(2)
    streams = [torch.cuda.Stream() for _ in range(2)]
    own = [dict(stream=s, workspace=_workspace()) for s in streams]
    for i in range(2):
        calls.run(i)
    want = calls.take()
    graphs = []
    for i, s in enumerate(streams):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=s):
            calls.run(i, **own[i])
    for eager in (True, False, True, False):
        for _ in range(3):
            for i, s in enumerate(streams):
                if eager:
                    calls.run(i, **own[i])
                else:
                    with torch.cuda.stream(s):
                        graphs[i].replay()
        for got, expected in zip(calls.take(), want):
            for t, u in zip(got, expected):
                assert torch.equal(t, u)
