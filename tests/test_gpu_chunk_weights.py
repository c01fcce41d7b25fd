"""Chunks whose weights lie far apart: one key that leads all others (an attention sink, as a rule the context's first token), logits that rise along
the context, values of any size.  A light key's weight and its value's codes have to come through as well as a heavy one's.  Bounds: those of the chunk
operator's own tests, relative to what the keys contribute; the leading key's value is zero, so that the others are all of the output."""
import math

import numpy as np
import pytest
import torch

from oracle import gkv_oracle as O
from paper_2608_23599_b200 import binding as B
from tests.test_gpu_chunk import check, f32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EXT = dict(policy=B.POLICY_EXTERNAL)


def streams_alike(k, v, levels, batch, n_kv, group):
    """A cache whose streams all hold the rows k, v [ctx][128], and the oracle's of one such stream."""
    ctx = k.shape[0]
    oc = O.GradedCache(O.Config(n_layers=1, batch=1, n_q_heads=group, n_kv_heads=1, d_k=128, d_v=128, max_ctx=ctx + 64, **EXT))
    oc.append_demote(0, f32(k)[None, :, None], f32(v)[None, :, None], None, levels[None, None])
    c = B.Cache(B.make_config(1, batch, group * n_kv, n_kv, 128, 128, ctx + 64, **EXT))
    spread = [x.to(DEV)[None, :, None].expand(batch, ctx, n_kv, 128).contiguous() for x in (k, v)]
    c.gkv_append_demote(0, *spread, level_plan=np.broadcast_to(levels, (batch, n_kv, len(levels))).copy())
    return c, oc


def run_alike(c, oc, q, k, v, batch, n_kv):
    """q, k, v: [n_new][heads][128] of one stream.  Every stream has to give the same bits but for where it was cut."""
    n_new, group, _ = q.shape
    dq = q.to(DEV)[None, :, None].expand(batch, n_new, n_kv, group, 128).reshape(batch, n_new, n_kv * group, 128).contiguous()
    dk, dv = (x.to(DEV)[None].expand(batch, n_new, n_kv, 128).contiguous() for x in (k, v))
    out = torch.full(dq.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full(dq.shape[:3], 7.0, device=DEV)
    c.gkv_chunk_attn(0, dq, dk, dv, out, lse=lse)
    torch.cuda.synchronize()
    c.gkv_bits_report(0)
    seen = {}
    for b in range(batch):
        for h in range(n_kv):
            o, l = out[b, :, h * group:(h + 1) * group], lse[b, :, h * group:(h + 1) * group]
            key = o.float().cpu().numpy().tobytes() + l.cpu().numpy().tobytes()
            if key not in seen:
                seen[key] = True
                check(o[None], l[None], oc, q[None], k[None], v[None])
    return out, lse


def beyond_the_format(c, v, level):
    """Values whose scales no read takes (above 4094) or that are beyond fp16: the cache says so, and nothing is asked of what is read from it."""
    g = v.float().view(v.shape[0], 4, 32)
    beyond = float((g.amax(-1) - g.amin(-1)).max()) / (2 ** level - 1) > 4094.0 or float(g.abs().max()) > 65504.0
    assert B.load().gkv_bits_report(c.handle, 0, B.C.byref(B.GkvBits())) == (B.ERR_RANGE if beyond else B.OK)
    return beyond


def sink(ctx, n_new, group, lead, gain, noise=0.3, seed=0):
    """Rows whose first key leads the others by `lead` nats for every query; its value is zero, the others' are of size `gain`."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(n_new, group, 128, generator=g) * noise
    k, v = torch.randn(ctx + n_new, 128, generator=g), gain * torch.randn(ctx + n_new, 128, generator=g)
    q[..., 0], k[:, 0] = 8.0, 0.0
    k[0], v[0] = 0.0, 0.0
    k[0, 0] = lead * math.sqrt(128.0) / 8.0
    q, k, v = q.bfloat16(), k.bfloat16(), v.bfloat16()
    return k[:ctx], v[:ctx], (q, k[ctx:, None], v[ctx:, None])


def plan(ctx, level, first=16):
    return np.array([first] + [level] * (ctx // 64 - 1), dtype=np.int8)


@pytest.mark.parametrize("level", [8, 4, 2])
@pytest.mark.parametrize("gain", [1.0, 0.1, 0.02])
@pytest.mark.parametrize("lead,noise", [(11.0, 0.3), (13.0, 0.0), (16.0, 0.0)])
def test_a_leading_key_and_few_rows(level, gain, lead, noise):
    """More streams than CTAs, 64 rows: the team that meets the leading key reads a third of the context."""
    ctx, batch, n_kv = 64 * 48, 20, 8
    k, v, x = sink(ctx, 16, 4, lead, gain, noise, seed=level)
    c, oc = streams_alike(k, v, plan(ctx, level), batch, n_kv, 4)
    run_alike(c, oc, *x, batch, n_kv)


@pytest.mark.parametrize("level", [8, 4, 2])
@pytest.mark.parametrize("n_new", [1, 5])
def test_a_leading_key_and_a_long_context_of_few_streams(level, n_new):
    ctx = 64 * 500 + 7
    k, v, x = sink(ctx, n_new, 4, 13.0, 0.1, 0.1, seed=level)
    c, oc = streams_alike(k, v, plan(ctx, level), 1, 2, 4)
    run_alike(c, oc, *x, 1, 2)


@pytest.mark.parametrize("level", [8, 4, 2])
def test_the_leading_key_is_stored_as_codes(level):
    ctx = 64 * 40
    k, v, x = sink(ctx, 16, 4, 8.0, 0.1, 0.2, seed=level)
    c, oc = streams_alike(k, v, plan(ctx, level, first=level), 20, 8, 4)
    run_alike(c, oc, *x, 20, 8)


@pytest.mark.parametrize("level", [8, 4, 2])
@pytest.mark.parametrize("n_new", [4, 16, 40])
def test_logits_that_rise_and_fall_along_the_context(level, n_new):
    """From -15 to 15 nats and back: the reference moves all the way up, and what comes behind it is light."""
    ctx = 64 * 60
    g = torch.Generator().manual_seed(level)
    q, k, v = 0.2 * torch.randn(n_new, 4, 128, generator=g), torch.randn(ctx + n_new, 128, generator=g), 0.1 * torch.randn(ctx + n_new, 128, generator=g)
    q[..., 0], k[:, 0] = 8.0, 0.0
    k[:ctx, 0] = (15.0 - 30.0 * torch.linspace(-1, 1, ctx).abs()) * math.sqrt(128.0) / 8.0
    q, k, v = q.bfloat16(), k.bfloat16(), v.bfloat16()
    c, oc = streams_alike(k[:ctx], v[:ctx], plan(ctx, level, first=level), 20, 8, 4)
    run_alike(c, oc, q, k[ctx:, None], v[ctx:, None], 20, 8)


@pytest.mark.parametrize("level", [8, 4])
@pytest.mark.parametrize("far", [0, 17])
def test_values_of_very_different_sizes(level, far):
    """A block with values of 20,000 that hardly counts, among values of 0.02."""
    ctx = 64 * 40
    k, v, x = sink(ctx, 16, 4, 9.0, 0.02, 0.2, seed=level)
    k, v = k.clone(), v.clone()
    at = 64 * (1 + far)
    k[at:at + 64, 0] = -40.0 * math.sqrt(128.0) / 8.0
    v[at:at + 64] = (v[at:at + 64].float() * 1e6).bfloat16()
    c, oc = streams_alike(k, v, plan(ctx, level), 20, 8, 4)
    if not beyond_the_format(c, v[64:], level):
        run_alike(c, oc, *x, 20, 8)


@pytest.mark.parametrize("level", [8, 4, 2])
@pytest.mark.parametrize("gain", [4000.0, 1e-3])
def test_large_and_small_values(level, gain):
    """Up to the largest scales that the read path takes, and small ones."""
    ctx = 64 * 20
    k, v, x = sink(ctx, 16, 4, 3.0, gain, 0.3, seed=level)
    c, oc = streams_alike(k, v, plan(ctx, level), 20, 8, 4)
    if not beyond_the_format(c, v[64:], level):
        run_alike(c, oc, *x, 20, 8)


@pytest.mark.parametrize("level", [16, 8, 4, 2])
@pytest.mark.parametrize("lead,noise", [(11.0, 0.3), (13.0, 0.0), (14.5, 0.0)])
def test_a_leading_key_and_many_rows(level, lead, noise):
    ctx = 64 * 130 + 5
    k, v, x = sink(ctx, 40, 4, lead, 1.0, noise, seed=level)
    c, oc = streams_alike(k, v, plan(ctx, level), 1, 2, 4)
    run_alike(c, oc, *x, 1, 2)
