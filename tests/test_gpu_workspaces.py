"""Kept workspaces that have to grow: the small one is given back before the large one is asked for."""
import numpy as np
import pytest
import torch

from paper_2608_23599_b200 import binding as B
from tests import test_gpu_chunk as tc
from tests import test_gpu_prompt as tp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROUNDING = 2 << 20              # torch's allocator hands out large blocks by steps of 2 MiB


def peak_over(call):
    """Bytes that torch's allocator handed out at most during the call, over those before it."""
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    call()
    torch.cuda.synchronize()
    return torch.cuda.max_memory_allocated() - before


def test_a_chunks_workspace_grows():
    c, oc, g = tc.caches(8, 2, 64 * 60, seed=1, plan=4, **tc.EXT)
    xs = [[t.to(DEV) for t in tc.chunk(g, 1, n, 8, 2)] for n in (100, 900)]
    outs = [torch.empty_like(x[0]) for x in xs]
    small, large = (c.gkv_chunk_workspace_bytes(0, x[0].shape[1]) for x in xs)
    c.gkv_chunk_attn(0, *xs[0], outs[0])
    assert 2 * ROUNDING < small < large
    assert peak_over(lambda: c.gkv_chunk_attn(0, *xs[1], outs[1])) <= large - small + ROUNDING


def test_a_prompts_workspace_grows():
    B._prompt_spaces.clear()
    small, large = (tp.make([n], 8, 2, seed=n) for n in (1300, 2500))
    outs = [torch.empty_like(x[0]) for x in (small, large)]
    B.gkv_prompt_attn(*small[:3], outs[0], small[3])
    held = sum(kept[1] for kept in B._prompt_spaces.values())
    grown = peak_over(lambda: B.gkv_prompt_attn(*large[:3], outs[1], large[3]))
    need = sum(kept[1] for kept in B._prompt_spaces.values())
    assert 2 * ROUNDING < held < need and grown <= need - held + ROUNDING
