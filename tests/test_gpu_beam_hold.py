"""Searches whose pool runs out: groups wait for pages and go on, step by step and in a captured graph."""
import pytest
import torch

import beam_story

pytestmark = pytest.mark.gpu


def _captured(r):
    logits = torch.zeros((len(r.lens), beam_story.VOCAB), device="cuda")
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        r.step(logits)

    def step(x):
        logits.copy_(x)
        graph.replay()
    return step


def test_groups_that_wait_for_pages_go_on_as_they_were():
    def make(n):
        return beam_story.runner(4, 3, n, "cuda", hold=True)

    print("step by step", flush=True)
    waited = beam_story.waits_and_goes_on(make, lambda r: r.step)
    print("in a graph", flush=True)                              # (kernels are loaded by now)
    assert beam_story.waits_and_goes_on(make, _captured) == waited > 3
