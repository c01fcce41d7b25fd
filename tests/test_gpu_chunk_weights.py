"""Chunks whose weights lie far apart: one key that leads all others (an attention sink, as a rule the context's first token), logits that rise along
the context, values of any size.  A light key's weight and its value's codes have to come through as well as a heavy one's.  Bounds: those of the chunk
operator's own tests (logits, log-sum-exps, weights, values, output), relative to what the keys contribute; in most tests the leading key's value is
zero, so that the others are all of the output.  Weights are fp16 numbers over codes and where there are many rows, so that there is an end to that:
a number below 2^-14 is off by up to 2^-25.
  Few rows: 2^11 is the heaviest weight of an item of 32 keys, at most the row's heaviest.  A weight is off by 2^-36 of that, and what it multiplies
  (scale * code and the zero point) is at most three times the token's largest value.  The products of weights and scales have 2^14 at least where
  the item's heaviest weight and largest scale meet: off by 2^-39 of it, times a code, less than a quarter of the former for 8 bits and less.
  Many rows: 2^7 is the weight at the reference, which the row's heaviest reaches.  A weight is off by 2^-32 of that.
With 1.25 * 3 * 2^-36 * max_c |v_jc| and 2^-32 |v_jc| summed over the keys the output is off by that much more, in 32-bit terms nothing."""
import math

import numpy as np
import pytest
import torch

from oracle import gkv_oracle as O
from paper_2608_23599_b200 import binding as B
from tests.test_gpu_chunk import f32

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


def check(out, lse, oc, q, k, v):
    """One stream: out, lse, q [n_new][heads][.], k, v [n_new][128]."""
    n, group, _ = q.shape
    got, gl = out.float().cpu().double().numpy(), lse.cpu().double().numpy()
    q, k, v = (x.double().numpy() for x in (q, k, v))
    ck, cv = oc.reconstruct(oc.streams[(0, 0, 0)])
    kk, vv = np.concatenate([ck, k]), np.concatenate([cv, v])
    hide = np.arange(len(kk))[None] > len(ck) + np.arange(n)[:, None]
    seen = np.where(hide, 0.0, 1.0)
    floor = 2.0 ** -32 * (seen @ np.abs(vv)) if n * group > 64 else 3.75 * 2.0 ** -36 * (seen @ np.abs(vv).max(1))[:, None]
    num = den = lnum = lden = 0.0
    for a in range(group):
        x = np.where(hide, -np.inf, q[:, a] @ kk.T * oc.scale)
        mag = np.where(hide, 0, np.abs(q[:, a]) @ np.abs(kk.T) * oc.scale).max(1)
        top = x.max(1)
        rl = top + np.log(np.exp(x - top[:, None]).sum(1))
        w = np.exp(x - rl[:, None])
        o, ov = w @ vv, w @ np.abs(vv)
        slack = (2.0 ** -16 + 2.0 ** -21) * mag + 2.0 ** -20
        tol = (2 * slack[:, None] + 2.0 ** -8 + 2.0 ** -11) * ov + 2.0 ** -8 * np.abs(o) + floor
        err = np.abs(got[:, a] - o)
        assert (err <= tol * 1.01).all(), f"head {a}: off by {np.nanmax(err - tol):.3e} more than the bound"
        assert (np.abs(gl[:, a] - rl) <= slack + 2.0 ** -21 * np.abs(rl)).all(), f"head {a}: log-sum-exp off by {np.abs(gl[:, a] - rl).max():.3e}"
        num, den = num + (np.maximum(err - floor, 0) ** 2).sum(), den + (o ** 2).sum()
        lnum, lden = lnum + ((gl[:, a] - rl) ** 2).sum(), lden + (rl ** 2).sum()
    assert num <= (4e-3) ** 2 * den, f"off by {math.sqrt(num / den):.2e} of the norm"
    assert lnum <= (4e-6) ** 2 * lden, f"log-sum-exp off by {math.sqrt(lnum / lden):.2e} of its norm"


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
                check(o, l, oc, q, k[:, 0], v[:, 0])
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
    ctx, batch, n_kv = 64 * 50, 20, 8
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


@pytest.mark.parametrize("level", [8, 4, 2])
@pytest.mark.parametrize("lead", [13.7, 40.0])
@pytest.mark.parametrize("n_new", [6, 40])
def test_a_large_logit_over_codes(level, lead, n_new):
    """One channel makes the largest logit, of a key that is stored as codes and whose value counts."""
    ctx, at = 64 * 23 + 3, 272
    g = torch.Generator().manual_seed(level)
    q, k, v = 0.1 * torch.randn(n_new, 4, 128, generator=g), torch.randn(ctx + n_new, 128, generator=g), torch.randn(ctx + n_new, 128, generator=g)
    q[..., 0], k[:, 0], k[at] = 8.0, 0.0, 0.0
    k[at, 0] = lead * math.sqrt(128.0) / 8.0
    q, k, v = q.bfloat16(), k.bfloat16(), v.bfloat16()
    c, oc = streams_alike(k[:ctx], v[:ctx], plan(ctx, level, first=level), 1, 2, 4)
    run_alike(c, oc, q, k[ctx:, None], v[ctx:, None], 1, 2)
