"""Prompt attention and prompt token masses against the definition in 64 bits, and in front of a bulk ingest.

Bounds.  A weight enters the value product as bf16 (off by at most eps / 2 = 2^-8 of itself), the output is rounded once more:
|out - o| <= 2^-8 (sum_j w_j |v_j| + |o|), plus what 32-bit arithmetic leaves: a logit is a sum of 128 products, each addition
off by at most 2^-23 of the running sum of magnitudes A = scale * sum_c |q_c k_c|, so by at most 2^-16 A; the exponent's argument
and the function itself add a few 2^-22.  The log-sum-exp inherits the logits' error and its own rounding.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_23599_b200 import binding as B

pytestmark = pytest.mark.gpu
HEADS = [(8, 2), (8, 8), (4, 1), (16, 2), (6, 2), (5, 1), (12, 2), (7, 1)]


def make(lengths, n_q, n_kv, seed=0, gain=8.0, dev="cuda:0", lead=0, behind=0, fused=False, garbage=False):
    """Packed rows with `lead` rows in front and `behind` behind (of NaN and infinities where `garbage`)."""
    g = torch.Generator().manual_seed(seed)
    t = lead + sum(lengths) + behind
    q, k, v = torch.randn(t, n_q, 128, generator=g), torch.randn(t, n_kv, 128, generator=g), torch.randn(t, n_kv, 128, generator=g)
    k[:, :, :4] *= gain
    if garbage:
        for x in (q, k, v):
            x[:lead], x[t - behind:] = math.nan, math.inf
    q, k, v = (x.bfloat16().to(dev) for x in (q, k, v))
    if fused:
        z = torch.cat([q, k, v], 1)
        q, k, v = z[:, :n_q], z[:, n_q:n_q + n_kv], z[:, n_q + n_kv:]
    off = lead + np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    return q, k, v, off


def reference(q, k, v, off, scale=None):
    """out, sum_j w_j |v_j|, lse, max_j scale sum_c |q_c k_jc| in 64 bits; rows of no sequence are zero."""
    scale = scale or 1.0 / math.sqrt(128.0)
    t, n_q, _ = q.shape
    g = n_q // k.shape[1]
    o, ov = torch.zeros(t, n_q, 128, dtype=torch.float64, device=q.device), torch.zeros(t, n_q, 128, dtype=torch.float64, device=q.device)
    lse, mag = torch.zeros(t, n_q, dtype=torch.float64, device=q.device), torch.zeros(t, n_q, dtype=torch.float64, device=q.device)
    for a, b in zip(off[:-1].tolist(), off[1:].tolist()):
        if a == b:
            continue
        hide = torch.ones(b - a, b - a, dtype=torch.bool, device=q.device).triu(1)
        for h in range(n_q):
            qq, kk, vv = q[a:b, h].double(), k[a:b, h // g].double(), v[a:b, h // g].double()
            x = ((qq @ kk.T) * scale).masked_fill(hide, -math.inf)
            lse[a:b, h] = torch.logsumexp(x, 1)
            w = torch.exp(x - lse[a:b, h, None])
            o[a:b, h], ov[a:b, h] = w @ vv, w @ vv.abs()
            mag[a:b, h] = ((qq.abs() @ kk.abs().T) * scale).masked_fill(hide, 0).amax(1)
    return o, ov, lse, mag


def check(out, lse, ref, rows):
    o, ov, rl, mag = (x[rows] for x in ref)
    slack = 2.0 ** -16 * mag + 2.0 ** -20
    tol = 2.0 ** -8 * (ov + o.abs()) * (1 + 2.0 ** -7) + 2 * slack[..., None] * ov
    bad = (out[rows].double() - o).abs() - tol
    worst = float(bad.max())
    assert worst <= 0, f"output off by {worst:.3e} more than the bound"
    bad = (lse[rows].double() - rl).abs() - (slack + 2.0 ** -22 * rl.abs())
    worst = float(bad.max())
    assert worst <= 0, f"log-sum-exp off by {worst:.3e} more than the bound"


def run(q, k, v, off, **kw):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=q.device)
    lse = torch.full(q.shape[:2], 7.0, device=q.device)
    B.gkv_prompt_attn(q, k, v, out, off, lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("n_q,n_kv", HEADS)
def test_one_sequence_of_every_group_size(n_q, n_kv):
    q, k, v, off = make([300], n_q, n_kv, seed=n_q)
    check(*run(q, k, v, off), reference(q, k, v, off), slice(0, 300))


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 640, 1025])
def test_lengths_around_tile_edges(n):
    q, k, v, off = make([n], 8, 2, seed=n)
    check(*run(q, k, v, off), reference(q, k, v, off), slice(0, n))


def test_one_token_returns_its_value():
    q, k, v, off = make([1, 1, 1], 8, 2)
    out, _ = run(q, k, v, off)
    assert torch.equal(out, v.repeat_interleave(4, 1))


@pytest.mark.parametrize("fused", [False, True])
def test_packed_sequences(fused):
    lengths = [5, 0, 130, 1, 257, 64, 0, 33]
    q, k, v, off = make(lengths, 12, 4, seed=3, fused=fused)
    check(*run(q, k, v, off), reference(q, k, v, off), slice(0, sum(lengths)))


def test_rows_of_no_sequence_are_neither_used_nor_written():
    lengths = [70, 200]
    q, k, v, off = make(lengths, 8, 2, seed=4, lead=9, behind=13, garbage=True)
    out, lse = run(q, k, v, off)
    n = sum(lengths)
    z = [torch.nan_to_num(x, nan=0.0, posinf=0.0) for x in (q, k, v)]
    check(out, lse, reference(*z, off), slice(9, 9 + n))
    assert bool((out[:9] == 7).all()) and bool((out[9 + n:] == 7).all()) and bool((lse[:9] == 7).all()) and bool((lse[9 + n:] == 7).all())


def test_strided_output_and_scale():
    q, k, v, off = make([150], 8, 2, seed=5)
    wide = torch.full((150, 12, 128), 7.0, dtype=torch.bfloat16, device=q.device)
    lse = torch.empty(150, 8, device=q.device)
    B.gkv_prompt_attn(q, k, v, wide[:, 2:10], off, lse=lse, softmax_scale=0.03)
    check(wide[:, 2:10], lse, reference(q, k, v, off, 0.03), slice(0, 150))
    assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 10:] == 7).all())


def test_logits_far_apart_and_a_rising_maximum():
    """Keys that grow along the sequence move the softmax reference in almost every step."""
    q, k, v, off = make([900], 4, 1, seed=6, gain=1.0)
    k = (k.float() * torch.linspace(0.1, 40.0, 900, device=k.device)[:, None, None]).bfloat16()
    check(*run(q, k, v, off), reference(q, k, v, off), slice(0, 900))


def test_more_sequences_than_one_launch_takes():
    lengths = [1 + i % 3 for i in range(1030)]
    q, k, v, off = make(lengths, 4, 2, seed=7)
    check(*run(q, k, v, off), reference(q, k, v, off), slice(0, sum(lengths)))


def test_same_bits_every_time_and_on_another_stream():
    q, k, v, off = make([700, 90], 16, 2, seed=8)
    first = run(q, k, v, off)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(q, k, v, off)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_captured_and_replayed():
    q, k, v, off = make([333, 40], 8, 2, seed=9)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=q.device)
    mass = torch.zeros(373 * 2, device=q.device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gkv_prompt_attn(q, k, v, out, off, lse=lse)
        B.gkv_prompt_mass(q, k, lse, mass, off, 16)
    q.copy_(torch.randn_like(q.float()).bfloat16())
    graph.replay()
    torch.cuda.synchronize()
    ref = reference(q, k, v, off)
    check(out, lse, ref, slice(0, 373))
    check_mass(mass, q, k, off, 16, ref)


# ---- masses ----
def check_mass(mass, q, k, off, n_obs, ref, scale=None):
    scale = scale or 1.0 / math.sqrt(128.0)
    n_kv, g = k.shape[1], q.shape[1] // k.shape[1]
    _, _, lse, mag = ref
    for a, b in zip(off[:-1].tolist(), off[1:].tolist()):
        if a == b:
            continue
        o, n = min(n_obs, b - a), b - a
        hide = torch.ones(o, n, dtype=torch.bool, device=q.device).triu(n - o + 1)
        got = mass[(a - int(off[0])) * n_kv:(b - int(off[0])) * n_kv].view(n_kv, n).double()
        for h in range(n_kv):
            want = torch.zeros(n, dtype=torch.float64, device=q.device)
            for x in range(h * g, h * g + g):
                s = ((q[b - o:b, x].double() @ k[a:b, h].double().T) * scale).masked_fill(hide, -math.inf)
                want += torch.exp(s - lse[b - o:b, x, None]).sum(0)
            want /= o * g
            # a weight is off by the logit's and the log-sum-exp's error, the sum by an addition's rounding per row
            rel = 2 * (2.0 ** -16 * float(mag[b - o:b].max()) + 2.0 ** -20 + 2.0 ** -22 * float(lse[b - o:b].abs().max())) + o * g * 2.0 ** -24
            assert float((got[h] - want).abs().max() / want.max()) <= rel
            assert bool(((got[h] - want).abs() <= rel * want + 1e-30).all())
            assert abs(float(got[h].sum()) - 1.0) <= rel + n * 2.0 ** -24


@pytest.mark.parametrize("n_q,n_kv", HEADS)
@pytest.mark.parametrize("n_obs", [1, 16, 37])
def test_masses(n_q, n_kv, n_obs):
    lengths = [301, 0, 8, 128, 1]
    q, k, v, off = make(lengths, n_q, n_kv, seed=n_q + n_obs)
    _, lse = run(q, k, v, off)
    mass = torch.full((sum(lengths) * n_kv,), 7.0, device=q.device)
    B.gkv_prompt_mass(q, k, lse, mass, off, n_obs)
    check_mass(mass, q, k, off, n_obs, reference(q, k, v, off))


@pytest.mark.parametrize("n,n_obs", [(2000, 16), (513, 300), (129, 10 ** 6), (257, 257)])
def test_masses_of_many_rows(n, n_obs):
    """More observing rows than one product has columns, and more tiles than one CTA takes."""
    q, k, v, off = make([n], 8, 2, seed=n, lead=3)
    _, lse = run(q, k, v, off)
    mass = torch.zeros(n * 2, device=q.device)
    B.gkv_prompt_mass(q, k, lse, mass, off, n_obs)
    check_mass(mass, q, k, off, n_obs, reference(q, k, v, off))


def test_masses_of_many_tiles():
    q, k, v, off = make([40000], 4, 4, seed=2, gain=4.0)
    lse = torch.zeros(40000, 4, device=q.device)
    for h in range(4):
        lse[-16:, h] = torch.logsumexp((q[-16:, h].double() @ k[:, h].double().T / math.sqrt(128.0)).masked_fill(
            torch.ones(16, 40000, dtype=torch.bool, device=q.device).triu(40000 - 15), -math.inf), 1).float()
    mass = torch.zeros(4 * 40000, device=q.device)
    B.gkv_prompt_mass(q, k, lse, mass, off, 16)
    mag = torch.zeros(40000, 4, dtype=torch.float64, device=q.device)
    mag[-16:] = 60.0
    check_mass(mass, q, k, off, 16, (None, None, lse.double(), mag))


def test_prompt_to_decode():
    """Attention, masses, ingest under the rate-distortion policy, and a decode step, as a serving program strings them together."""
    n, n_q, n_kv, b = 1000, 8, 2, 2
    q, k, v, off = make([n] * b, n_q, n_kv, seed=11)
    out, lse = run(q, k, v, off)
    mass = torch.empty(b, n_kv, n, device=q.device)
    B.gkv_prompt_mass(q, k, lse, mass, off, 16)
    ref = reference(q, k, v, off)
    check(out, lse, ref, slice(0, b * n))
    c = B.Cache(B.make_config(1, b, n_q, n_kv, 128, 128, 2048, policy=B.POLICY_RD, retire_after=128, rd_budget_bpv=16.0, residual_fraction=0.02))
    c.gkv_append_demote(0, k.view(b, n, n_kv, 128), v.view(b, n, n_kv, 128), token_mass=mass)
    # at a budget of 16 bits everything stays exact: the newest query's decode is the prompt's last row
    dec = torch.empty(b, n_q, 128, device=q.device)
    last = q.view(b, n, n_q, 128)[:, -1].contiguous()
    c.gkv_decode_attn(0, last, dec)
    torch.cuda.synchronize()
    o, ov = ref[0].view(b, n, n_q, 128)[:, -1], ref[1].view(b, n, n_q, 128)[:, -1]
    assert bool(((dec.double() - out.view(b, n, n_q, 128)[:, -1].double()).abs() <= 2.0 ** -8 * (ov + o.abs()) * 1.01 + 2e-3).all())
    c.close()
