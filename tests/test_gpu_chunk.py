"""Attention of a chunk of new tokens over the graded cache, against the oracle's reconstruction of the cache in 64 bits.

Bounds.  A key is the cache's own (codes times a scaled query pair, or an fp16 pair: 2^-21 of itself and less), a logit a sum of 128
products: with A = max_j scale * sum_c |q_c k_jc| it is off by at most (2^-16 + 2^-21) A (each addition by 2^-23 of the running sum).  A value
is rounded to fp16 (2^-11), a weight to bf16 or fp16 (2^-8 at most) and the output to bf16 (2^-8 of itself), so it is off by at most
2 (2^-16 + 2^-21) A ov + (2^-8 + 2^-11) ov + 2^-8 |o| with ov = sum_j w_j |v_j|.  The log-sum-exp is off by (2^-16 + 2^-21) A and its own
rounding.  Roundings of this kind have no common sign: the whole output is within 4e-3 of its norm, the log-sum-exp within 4e-6.
"""
import math

import numpy as np
import pytest
import torch

from oracle import gkv_oracle as O
from paper_2608_23599_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rows(g, *shape, gain=1.0):
    x = torch.randn(*shape, generator=g)
    x[..., :4] *= gain
    return x.bfloat16()


def f32(t):
    return t.to(torch.float32).numpy()


def caches(n_q, n_kv, ctx, batch=1, seed=0, plan=None, max_ctx=None, **kw):
    """The library's cache and the oracle's, with the same rows; plan: levels of all blocks, or a function of (b, h, block)."""
    g = torch.Generator().manual_seed(seed)
    max_ctx = max_ctx or max(ctx + 200, 64)
    oc = O.GradedCache(O.Config(n_layers=1, batch=batch, n_q_heads=n_q, n_kv_heads=n_kv, d_k=128, d_v=128, max_ctx=max_ctx, **kw))
    c = B.Cache(B.make_config(1, batch, n_q, n_kv, 128, 128, max_ctx, **kw))
    if ctx:
        k, v = rows(g, batch, ctx, n_kv, 128, gain=6.0), rows(g, batch, ctx, n_kv, 128)
        levels = None
        if plan is not None:
            nb = ctx // 64
            levels = np.array([[[plan(b, h, i) if callable(plan) else plan for i in range(nb)] for h in range(n_kv)] for b in range(batch)], dtype=np.int8)
            levels = levels.reshape(batch, n_kv, nb)
        mass = None
        if kw.get("policy") == B.POLICY_RD or kw.get("residual_fraction"):
            mass = torch.softmax(1.5 * torch.randn(batch, n_kv, ctx, generator=g), -1)
        oc.append_demote(0, f32(k), f32(v), None if mass is None else mass.numpy(), levels)
        c.gkv_append_demote(0, k.to(DEV), v.to(DEV), token_mass=None if mass is None else mass.to(DEV), level_plan=levels)
    return c, oc, g


def chunk(g, batch, n_new, n_q, n_kv):
    return rows(g, batch, n_new, n_q, 128), rows(g, batch, n_new, n_kv, 128, gain=6.0), rows(g, batch, n_new, n_kv, 128)


def run(c, q, k, v, lengths=None, **kw):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full(q.shape[:3], 7.0, device=DEV)
    c.gkv_chunk_attn(0, q.to(DEV), k.to(DEV), v.to(DEV), out, lse=lse, lengths=lengths, **kw)
    torch.cuda.synchronize()
    c.gkv_bits_report(0)               # (raises where a kernel gave up a wait)
    return out, lse


def check(out, lse, oc, q, k, v, lengths=None):
    batch, n_new, n_q, _ = q.shape
    n_kv = k.shape[2]
    scale = oc.scale
    got, gl = out.float().cpu().double().numpy(), lse.cpu().double().numpy()
    q, k, v = (x.double().numpy() for x in (q, k, v))
    num = den = lnum = lden = 0.0
    for b in range(batch):
        n = n_new if lengths is None else int(lengths[b])
        assert (got[b, n:] == 7).all() and (gl[b, n:] == 7).all(), "rows behind a sequence's last one were written"
        for h in range(n_kv if n else 0):
            ck, cv = oc.reconstruct(oc.streams[(0, b, h)]) if oc.streams[(0, b, h)].ctx else (np.zeros((0, 128)), np.zeros((0, 128)))
            kk, vv = np.concatenate([ck, k[b, :n, h]]), np.concatenate([cv, v[b, :n, h]])
            hide = np.arange(len(kk))[None] > len(ck) + np.arange(n)[:, None]
            for a in range(h * n_q // n_kv, (h + 1) * n_q // n_kv):
                x = np.where(hide, -np.inf, q[b, :n, a] @ kk.T * scale)
                mag = np.where(hide, 0, np.abs(q[b, :n, a]) @ np.abs(kk.T) * scale).max(1)
                top = x.max(1)
                rl = top + np.log(np.exp(x - top[:, None]).sum(1))
                w = np.exp(x - rl[:, None])
                o, ov = w @ vv, w @ np.abs(vv)
                slack = (2.0 ** -16 + 2.0 ** -21) * mag + 2.0 ** -20
                tol = (2 * slack[:, None] + 2.0 ** -8 + 2.0 ** -11) * ov + 2.0 ** -8 * np.abs(o)
                err = np.abs(got[b, :n, a] - o)
                assert (err <= tol * 1.01).all(), f"sequence {b} head {a}: off by {np.nanmax(err - tol):.3e} more than the bound"
                assert (np.abs(gl[b, :n, a] - rl) <= slack + 2.0 ** -21 * np.abs(rl)).all(), f"sequence {b} head {a}: log-sum-exp off by {np.abs(gl[b, :n, a] - rl).max():.3e}"
                num, den = num + (err ** 2).sum(), den + (o ** 2).sum()
                lnum, lden = lnum + ((gl[b, :n, a] - rl) ** 2).sum(), lden + (rl ** 2).sum()
    assert lnum <= (4e-6) ** 2 * lden, f"log-sum-exp off by {math.sqrt(lnum / lden):.2e} of its norm"
    assert num <= (4e-3) ** 2 * den, f"off by {math.sqrt(num / den):.2e} of the norm"


EXT = dict(policy=B.POLICY_EXTERNAL)


@pytest.mark.parametrize("level", [16, 8, 4, 2, 1])
@pytest.mark.parametrize("n_new", [1, 5, 9, 17, 40])
def test_every_rung(level, n_new):
    c, oc, g = caches(8, 2, 64 * 7 + 13, seed=level + n_new, plan=level, **EXT)
    x = chunk(g, 1, n_new, 8, 2)
    check(*run(c, *x), oc, *x)


@pytest.mark.parametrize("n_q,n_kv", [(8, 8), (4, 1), (16, 2), (6, 2), (5, 1), (12, 2), (7, 1), (2, 1)])
@pytest.mark.parametrize("n_new", [3, 21])
def test_group_sizes_over_a_mixed_plan(n_q, n_kv, n_new):
    plan = lambda b, h, i: [16, 4, 2, 1, 8, 4, 1][(3 * i + h + b) % 7]
    c, oc, g = caches(n_q, n_kv, 64 * 20 + 1, batch=2, seed=n_q, plan=plan, **EXT)
    x = chunk(g, 2, n_new, n_q, n_kv)
    check(*run(c, *x), oc, *x)


@pytest.mark.parametrize("ctx", [0, 1, 63, 64, 65, 128])
@pytest.mark.parametrize("n_new", [1, 2, 33, 65, 130])
def test_short_contexts(ctx, n_new):
    c, oc, g = caches(8, 2, ctx, seed=ctx, plan=4, **EXT)
    x = chunk(g, 1, n_new, 8, 2)
    check(*run(c, *x), oc, *x)


@pytest.mark.parametrize("n_new", [4, 50])
def test_many_centroids(n_new):
    """More centroid blocks than one step takes, alone and among others."""
    plan = lambda b, h, i: 1 if i % 9 else 4
    c, oc, g = caches(8, 2, 64 * 190 + 5, seed=3, plan=plan, **EXT)
    x = chunk(g, 1, n_new, 8, 2)
    check(*run(c, *x), oc, *x)


@pytest.mark.parametrize("n_new", [1, 6, 40])
@pytest.mark.parametrize("fraction", [0.02, 0.15])
def test_residual_rows(n_new, fraction):
    """Exact residual rows take the place of their stored copies, in centroid blocks too."""
    kw = dict(policy=B.POLICY_RD, rd_budget_bpv=4.0, retire_after=64, residual_fraction=fraction)
    c, oc, g = caches(8, 2, 64 * 30 + 9, batch=2, seed=7, **kw)
    levels = np.concatenate([oc.levels(0, b, h) for b in range(2) for h in range(2)])
    assert (levels < 16).any()
    x = chunk(g, 2, n_new, 8, 2)
    check(*run(c, *x), oc, *x)


def test_centroid_blocks_with_residual_rows():
    kw = dict(policy=B.POLICY_STAIRCASE, stair_tokens=(64, 0, 0, 0), residual_fraction=0.3)
    c, oc, g = caches(8, 2, 64 * 12 + 9, seed=8, **kw)
    x = chunk(g, 1, 7, 8, 2)
    check(*run(c, *x), oc, *x)


@pytest.mark.parametrize("lengths", [[5, 0, 3], [0, 0, 1], [1, 5, 4]])
def test_lengths_of_drafts(lengths):
    c, oc, g = caches(8, 2, 64 * 9 + 30, batch=3, seed=9, plan=4, **EXT)
    x = chunk(g, 3, 5, 8, 2)
    check(*run(c, *x, lengths=lengths), oc, *x, lengths=lengths)


@pytest.mark.parametrize("lengths", [[300, 0], [1, 257], [64, 128]])
def test_lengths_of_messages(lengths):
    c, oc, g = caches(8, 2, 64 * 9 + 30, batch=2, seed=10, plan=8, **EXT)
    x = chunk(g, 2, 300, 8, 2)
    check(*run(c, *x, lengths=lengths), oc, *x, lengths=lengths)


def test_no_rows_at_all():
    c, oc, g = caches(8, 2, 100, batch=2, seed=10, plan=8, **EXT)
    x = chunk(g, 2, 3, 8, 2)
    out, lse = run(c, *x, lengths=[0, 0])
    assert bool((out == 7).all()) and bool((lse == 7).all())


def test_values_behind_a_sequence_may_be_anything():
    c, oc, g = caches(8, 2, 64 * 3 + 5, batch=2, seed=11, plan=4, **EXT)
    q, k, v = chunk(g, 2, 70, 8, 2)
    lengths = [66, 20]
    dirty = [t.clone() for t in (q, k, v)]
    for t in dirty:
        for b, n in enumerate(lengths):
            t[b, n:] = math.nan
    check(*run(c, *dirty, lengths=lengths), oc, q, k, v, lengths=lengths)


def test_more_streams_than_ctas():
    plan = lambda b, h, i: [4, 1, 2][(i + b) % 3]
    c, oc, g = caches(4, 4, 64 * 5 + 2, batch=40, seed=12, plan=plan, **EXT)
    x = chunk(g, 40, 4, 4, 4)
    check(*run(c, *x), oc, *x)


def test_long_context_of_one_stream_over_all_ctas():
    plan = lambda b, h, i: [4, 2, 8, 1, 16][i % 5]
    c, oc, g = caches(4, 1, 64 * 700 + 31, seed=13, plan=plan, **EXT)
    x = chunk(g, 1, 3, 4, 1)
    check(*run(c, *x), oc, *x)


def test_verify_then_append():
    """Drafts are verified, the accepted ones appended (blocks close and are demoted), and the next drafts verified."""
    kw = dict(policy=B.POLICY_STAIRCASE, stair_tokens=(64, 128, 128, 64))
    c, oc, g = caches(8, 2, 64 * 8 + 60, batch=2, seed=14, **kw)
    for accepted in (3, 5, 1):
        x = chunk(g, 2, 5, 8, 2)
        check(*run(c, *x), oc, *x)
        for i in range(accepted):
            k, v = x[1][:, i:i + 1].contiguous(), x[2][:, i:i + 1].contiguous()
            oc.append_demote(0, f32(k), f32(v))
            c.gkv_append_demote(0, k.to(DEV), v.to(DEV))
    # a chunk of one token sees what a decode step sees once the token is appended
    q, k, v = chunk(g, 2, 1, 8, 2)
    out, lse = run(c, q, k, v)
    check(out, lse, oc, q, k, v)
    before = c.gkv_ctx_len(0)
    c.gkv_append_demote(0, k.to(DEV), v.to(DEV))
    assert c.gkv_ctx_len(0) == before + 1
    dec, dl = torch.empty(2, 8, 128, device=DEV), torch.empty(2, 8, device=DEV)
    c.gkv_decode_attn(0, q[:, 0].contiguous().to(DEV), dec, dl)
    torch.cuda.synchronize()
    assert float((dec - out[:, 0].float()).abs().max()) <= 0.02 and float((dl - lse[:, 0]).abs().max()) <= 2e-3


def test_rising_logits_move_the_reference():
    c, oc, g = caches(4, 1, 64 * 40, seed=15, plan=16, **EXT)
    q, k, v = chunk(g, 1, 200, 4, 1)
    k = (k.float() * torch.linspace(0.1, 30.0, 200)[None, :, None, None]).bfloat16()
    check(*run(c, q, k, v), oc, q, k, v)


def test_same_bits_every_time_other_stream_and_given_workspace():
    plan = lambda b, h, i: [4, 2, 8, 1, 16][i % 5]
    c, oc, g = caches(8, 2, 64 * 50 + 3, seed=16, plan=plan, **EXT)
    x = chunk(g, 1, 30, 8, 2)
    first = run(c, *x)
    ws = torch.empty(c.gkv_chunk_workspace_bytes(0, 30), dtype=torch.uint8, device=DEV)
    again = run(c, *x, workspace=ws)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = run(c, *x)
    c.stream_handle = side.cuda_stream
    by_handle = run(c, *x)
    for y in (again, other, by_handle):
        assert torch.equal(first[0], y[0]) and torch.equal(first[1], y[1])


def test_captured_and_replayed_with_workspaces_of_their_own():
    c, oc, g = caches(8, 2, 64 * 30 + 3, seed=17, plan=4, **EXT)
    xs = [chunk(g, 1, 6, 8, 2) for _ in range(2)]
    dev = [[t.to(DEV) for t in x] for x in xs]
    outs = [(torch.full(x[0].shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.full(x[0].shape[:3], 7.0, device=DEV)) for x in xs]
    graphs = []
    for d, (out, lse) in zip(dev, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.gkv_chunk_attn(0, *d, out, lse=lse)
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for x, (out, lse) in zip(xs, outs):
        check(out, lse, oc, *x)


def test_refusals_on_a_gpu():
    c, oc, g = caches(8, 2, 100, batch=2, seed=18, plan=8, **EXT)
    q, k, v = (t.to(DEV) for t in chunk(g, 2, 3, 8, 2))
    out = torch.empty_like(q)
    for bad in (dict(q=q[:1]), dict(k_new=k[:, :2]), dict(out=out.float()), dict(v_new=v.cpu()), dict(lengths=[1]), dict(q=q.transpose(1, 2).contiguous())):
        a = dict(dict(q=q, k_new=k, v_new=v, out=out), **bad)
        with pytest.raises(ValueError):
            c.gkv_chunk_attn(0, **a)
    for kw in (dict(lengths=[1, 4]), dict(lengths=[-1, 1]), dict(workspace=torch.empty(16, dtype=torch.uint8, device=DEV))):
        with pytest.raises(B.GkvError):
            c.gkv_chunk_attn(0, q, k, v, out, **kw)
    with pytest.raises(B.GkvError):
        c.gkv_chunk_attn(1, q, k, v, out)
    m = B.Cache(B.make_config(1, 1, 16, 1, 576, 512, 256, v_aliases_k=1))
    n = B.C.c_size_t(0)
    assert B.load().gkv_chunk_workspace_bytes(m.handle, 0, 4, B.C.byref(n)) == B.ERR_UNSUPPORTED
    assert B.load().gkv_chunk_attn(m.handle, 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), 1, None, out.data_ptr(), None, None, 0, None) == B.ERR_UNSUPPORTED
