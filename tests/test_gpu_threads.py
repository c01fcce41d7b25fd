"""Prompts and chunks called by two host threads on one stream, whose workspace both use."""
import threading

import pytest
import torch

from paper_2608_23599_b200 import binding as B
from tests import test_gpu_chunk as tc
from tests import test_gpu_prompt as tp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def together(*calls):
    """Each call(i) 60 times in a thread of its own."""
    errors = []

    def run(call):
        try:
            for i in range(60):
                call(i)
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=run, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors


def test_two_threads_with_prompts_that_are_cut():
    sets = [tp.make([n], 8, 2, seed=n) for n in (2500, 2300)]
    want = [tp.run(*s) for s in sets]
    got = [[(torch.zeros_like(s[0]), torch.zeros(s[0].shape[:2], device=DEV)) for _ in range(60)] for s in sets]
    together(*(lambda i, s=s, g=g: B.gkv_prompt_attn(*s[:3], g[i][0], s[3], lse=g[i][1]) for s, g in zip(sets, got)))
    for w, g in zip(want, got):
        assert all(torch.equal(w[0], o) and torch.equal(w[1], l) for o, l in g)


@pytest.mark.parametrize("n_new", [5, 90])
def test_two_threads_with_chunks_of_one_cache(n_new):
    c, oc, g = tc.caches(8, 2, 64 * 60 + 9, seed=n_new, plan=4, **tc.EXT)
    sets = [tc.chunk(g, 1, n_new, 8, 2) for _ in range(2)]
    want = [tc.run(c, *x) for x in sets]
    sets = [[t.to(DEV) for t in x] for x in sets]
    got = [[(torch.zeros_like(x[0]), torch.zeros(x[0].shape[:3], device=DEV)) for _ in range(60)] for x in sets]
    together(*(lambda i, x=x, g=g: c.gkv_chunk_attn(0, *x, g[i][0], lse=g[i][1]) for x, g in zip(sets, got)))
    for w, g in zip(want, got):
        assert all(torch.equal(w[0], o) and torch.equal(w[1], l) for o, l in g)
