"""Prompt and chunk attention along the ways that lead to them: through the extension and through ctypes, with and without workspace, at the border
between the two chunk kernels, in graphs that are replayed in turn, with rows and strides that are refused, and as one run from a prompt to a
decode step.  Bounds: those of the two operators' own tests."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2608_23599_b200 import binding as B
from tests import test_gpu_chunk as tc
from tests import test_gpu_prompt as tp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EXT = dict(policy=B.POLICY_EXTERNAL)


def describe(q, k, off):
    d = B.GkvPrompt()
    d.struct_size, d.abi_version = C.sizeof(B.GkvPrompt), B.GKV_ABI_VERSION
    d.n_seqs, d.n_q_heads, d.n_kv_heads, d.head_dim, d.offsets = len(off) - 1, q.shape[1], k.shape[1], 128, off.ctypes.data
    return d


# ---- prompts ----
@pytest.mark.parametrize("as_given", [list, tuple, lambda o: np.asarray(o, dtype=np.int64), lambda o: torch.tensor(np.asarray(o))])
def test_offsets_of_any_kind(as_given):
    """An int32 array goes through the extension, everything else through ctypes: the same bits."""
    q, k, v, off = tp.make([200, 0, 77], 8, 2, seed=21)
    one, two = tp.run(q, k, v, off), tp.run(q, k, v, as_given(off))
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    masses = [torch.zeros(277 * 2, device=DEV) for _ in range(2)]
    B.gkv_prompt_mass(q, k, one[1], masses[0], off, 16)
    B.gkv_prompt_mass(q, k, one[1], masses[1], as_given(off), 16)
    assert torch.equal(*masses)


@pytest.mark.parametrize("lengths,n_q,n_kv", [([2500], 8, 2), ([1700, 1, 300], 16, 2), ([129] * 9 + [2049], 4, 4), ([1281], 7, 1)])
def test_cut_and_whole_tiles(lengths, n_q, n_kv):
    """Without the workspace that the call asks for tiles stay whole; with it they are cut into ranges that are merged."""
    q, k, v, off = tp.make(lengths, n_q, n_kv, seed=22)
    ref = tp.reference(q, k, v, off)
    d = describe(q, k, off)
    need = C.c_size_t(0)
    assert B.load().gkv_prompt_workspace_bytes(C.byref(d), C.byref(need)) == B.OK and need.value > 0
    ws = torch.full((need.value,), 0xff, dtype=torch.uint8, device=DEV)      # (NaN, whatever is not written)
    for room in (0, need.value - 16, need.value):
        out, lse = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.full(q.shape[:2], 7.0, device=DEV)
        rc = B.load().gkv_prompt_attn(C.byref(d), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), ws.data_ptr() if room else None, room,
                                      torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert rc == B.OK
        tp.check(out, lse, ref, slice(0, int(off[-1])))


def test_no_log_sum_exp():
    q, k, v, off = tp.make([2500, 3], 8, 2, seed=23)
    with_lse = tp.run(q, k, v, off)[0]
    out = torch.empty_like(with_lse)
    B.gkv_prompt_attn(q, k, v, out, off)
    assert torch.equal(out, with_lse)


def test_keys_of_later_tokens_may_be_anything():
    """What the mask hides is selected away: rows in front of a broken key, and the masses of tokens before it, are as without it."""
    q, k, v, off = tp.make([400, 300], 8, 2, seed=24)
    out, lse = tp.run(q, k, v, off)
    bad = k.clone()
    bad[350:400], bad[399] = math.nan, math.inf
    o2, l2 = tp.run(q, bad, v, off)
    keep = list(range(350)) + list(range(400, 700))
    assert torch.equal(out[keep], o2[keep]) and torch.equal(lse[keep], l2[keep])


def test_prompt_rows_that_are_refused():
    q, k, v, off = tp.make([64], 8, 2, seed=25)
    out = torch.empty_like(q)
    for bad in (dict(q=q[:1].expand(64, 8, 128)), dict(k=k[:1].expand(64, 2, 128)), dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(v=v[:, :1]),
                dict(k=k[:60], v=v[:60]), dict(out=out.half()), dict(q=q.cpu()), dict(off=[0, 65]), dict(off=[]), dict(off=[[0, 64]]),
                dict(lse=torch.zeros(8, 64, device=DEV).T), dict(lse=torch.zeros(64, 8, device=DEV, dtype=torch.float64))):
        a = dict(dict(q=q, k=k, v=v, out=out, off=off, lse=None), **bad)
        with pytest.raises(ValueError):
            B.gkv_prompt_attn(a["q"], a["k"], a["v"], a["out"], a["off"], lse=a["lse"])
    wide = torch.zeros(64, 8 * 128 + 4, device=DEV, dtype=torch.bfloat16)
    for bad in (dict(q=wide.as_strided((64, 8, 128), (1028, 128, 1))), dict(off=[0, 64, 30]), dict(off=[-1, 64])):
        a = dict(dict(q=q, off=off), **bad)
        with pytest.raises(B.GkvError):
            B.gkv_prompt_attn(a["q"], k, v, out, a["off"])
    lse = torch.zeros(64, 8, device=DEV)
    for m, n_obs, kind in ((torch.zeros(127, device=DEV), 16, ValueError), (torch.zeros(128, device=DEV), 0, B.GkvError), (torch.zeros(128), 4, ValueError),
                           (torch.zeros(256, device=DEV)[::2], 4, ValueError)):
        with pytest.raises(kind):
            B.gkv_prompt_mass(q, k, lse, m, off, n_obs)
    with pytest.raises(ValueError):
        B.gkv_prompt_mass(q, k, lse[:60], torch.zeros(128, device=DEV), off, 4)


def test_two_prompt_graphs_replayed_in_turn():
    """Each captured call has a workspace of its graph's own."""
    sets = [tp.make([2500], 8, 2, seed=s) for s in (26, 27)]
    outs, graphs = [], []
    for q, k, v, off in sets:
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.gkv_prompt_attn(q, k, v, out, off, lse=lse)
        outs.append((out, lse))
        graphs.append(graph)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
    torch.cuda.synchronize()
    for (q, k, v, off), got in zip(sets, outs):
        tp.check(*got, tp.reference(q, k, v, off), slice(0, 2500))


# ---- chunks ----
@pytest.mark.parametrize("as_given", [tuple, lambda o: np.asarray(o, dtype=np.int64), lambda o: np.asarray(o, dtype=np.int32), torch.tensor])
def test_lengths_of_any_kind(as_given):
    c, oc, g = tc.caches(8, 2, 64 * 5 + 9, batch=2, seed=31, plan=4, **EXT)
    for n_new, lengths in ((6, [6, 2]), (90, [71, 90])):
        x = tc.chunk(g, 2, n_new, 8, 2)
        one, two = tc.run(c, *x, lengths=lengths), tc.run(c, *x, lengths=as_given(lengths))
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
        tc.check(*one, oc, *x, lengths=lengths)


@pytest.mark.parametrize("n_q,n_kv,border", [(8, 2, 16), (8, 8, 64), (16, 2, 8), (5, 1, 12)])
def test_border_between_the_kernels(n_q, n_kv, border):
    plan = lambda b, h, i: [4, 2, 8, 1, 16][i % 5]
    c, oc, g = tc.caches(n_q, n_kv, 64 * 11 + 7, seed=32, plan=plan, **EXT)
    for n_new in (border, border + 1):
        x = tc.chunk(g, 1, n_new, n_q, n_kv)
        tc.check(*tc.run(c, *x), oc, *x)


def test_sequences_that_share_a_small_workspace():
    """Room for one sequence, and for two of three, at a time; below that the call is refused."""
    c, oc, g = tc.caches(8, 2, 64 * 6 + 5, batch=3, seed=33, plan=2, **EXT)
    x = tc.chunk(g, 3, 40, 8, 2)
    lengths = [40, 0, 33]
    all_three = c.gkv_chunk_workspace_bytes(0, 40)
    one = all_three
    while True:      # the smallest that is taken, to 64 KB
        try:
            tc.run(c, *x, lengths=lengths, workspace=torch.empty(one - 65536, dtype=torch.uint8, device=DEV))
        except B.GkvError:
            break
        one -= 65536
    assert one < all_three
    for room in (one, (one + all_three) // 2, all_three):
        ws = torch.full((room,), 0xff, dtype=torch.uint8, device=DEV)
        tc.check(*tc.run(c, *x, lengths=lengths, workspace=ws), oc, *x, lengths=lengths)


def test_many_rows_in_two_graphs_replayed_in_turn():
    c, oc, g = tc.caches(8, 2, 64 * 9 + 3, seed=34, plan=4, **EXT)
    xs = [tc.chunk(g, 1, 70, 8, 2) for _ in range(2)]
    dev = [[t.to(DEV) for t in x] for x in xs]
    outs = [(torch.zeros(x[0].shape, dtype=torch.bfloat16, device=DEV), torch.zeros(x[0].shape[:3], device=DEV)) for x in xs]
    graphs = []
    for d, (out, lse) in zip(dev, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.gkv_chunk_attn(0, *d, out, lse=lse)
        graphs.append(graph)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
    torch.cuda.synchronize()
    for x, got in zip(xs, outs):
        tc.check(*got, oc, *x)


def test_a_captured_call_on_a_stream_of_its_own_brings_its_workspace():
    c, oc, g = tc.caches(8, 2, 200, seed=35, plan=4, **EXT)
    x = tc.chunk(g, 1, 5, 8, 2)
    d = [t.to(DEV) for t in x]
    out, lse = torch.zeros(x[0].shape, dtype=torch.bfloat16, device=DEV), torch.zeros(x[0].shape[:3], device=DEV)
    ws = torch.empty(c.gkv_chunk_workspace_bytes(0, 5), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        c.stream_handle = torch.cuda.current_stream().cuda_stream
        with torch.cuda.stream(torch.cuda.Stream()):
            with pytest.raises(ValueError, match="workspace"):
                c.gkv_chunk_attn(0, *d, out, lse=lse)
            c.gkv_chunk_attn(0, *d, out, lse=lse, workspace=ws)
        c.stream_handle = None
    graph.replay()
    torch.cuda.synchronize()
    tc.check(out, lse, oc, *x)


@pytest.mark.parametrize("n_new", [6, 70])
def test_keys_of_later_new_tokens_may_be_anything(n_new):
    c, oc, g = tc.caches(8, 2, 64 * 3 + 9, seed=36, plan=4, **EXT)
    q, k, v = tc.chunk(g, 1, n_new, 8, 2)
    out, lse = tc.run(c, q, k, v)
    bad = k.clone()
    bad[:, -2:], bad[:, -1] = math.nan, math.inf
    o2, l2 = tc.run(c, q, bad, v)
    assert torch.equal(out[:, :-2], o2[:, :-2]) and torch.equal(lse[:, :-2], l2[:, :-2])


@pytest.mark.parametrize("n_new", [6, 70])
@pytest.mark.parametrize("ctx", [0, 64 * 40 + 9])
def test_a_broken_key_is_seen(n_new, ctx):
    """NaN comes through to every row that sees it, also where one of a stream's parts has it and the others have not."""
    c, oc, g = tc.caches(8, 2, ctx, seed=38, plan=4 if ctx else None, **EXT)
    q, k, v = tc.chunk(g, 1, n_new, 8, 2)
    out, lse = tc.run(c, q, k, v)
    bad = k.clone()
    bad[:, 3, :, 5] = math.nan
    o2, l2 = tc.run(c, q, bad, v)
    assert torch.equal(out[:, :3], o2[:, :3]) and torch.equal(lse[:, :3], l2[:, :3])
    assert bool(o2[:, 3:].isnan().all()) and bool(l2[:, 3:].isnan().all())


@pytest.mark.parametrize("n", [300, 2500])
def test_a_broken_key_of_a_prompt_is_seen(n):
    q, k, v, off = tp.make([n], 8, 2, seed=39)
    out, lse = tp.run(q, k, v, off)
    bad = k.clone()
    bad[100, :, 5] = math.nan
    o2, l2 = tp.run(q, bad, v, off)
    assert torch.equal(out[:100], o2[:100]) and torch.equal(lse[:100], l2[:100])
    assert bool(o2[100:].isnan().all()) and bool(l2[100:].isnan().all())


def test_calls_in_a_row_into_the_same_buffers():
    """Each kernel is launched while the one in front still runs: nothing is read or written before that one is done."""
    sets = [tp.make([900, 33], 8, 2, seed=s) for s in (41, 42)]
    off = sets[0][3]
    alone = []
    for q, k, v, _ in sets:
        out, lse = tp.run(q, k, v, off)
        mass = torch.zeros(933 * 2, device=DEV)
        B.gkv_prompt_mass(q, k, lse, mass, off, 40)
        alone.append((out, lse, mass))
    c, oc, g = tc.caches(8, 2, 64 * 20 + 5, seed=43, plan=4, **EXT)
    xs = [[t.to(DEV) for t in tc.chunk(g, 1, n, 8, 2)] for n in (6, 70, 6, 70)]
    chunks = []
    for x in xs:
        out, lse = torch.zeros_like(x[0]), torch.zeros(x[0].shape[:3], device=DEV)
        c.gkv_chunk_attn(0, *x, out, lse=lse)
        torch.cuda.synchronize()
        chunks.append((out, lse))
    q, k, v = (torch.empty_like(t.contiguous()) for t in sets[0][:3])
    out, lse, mass = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV), torch.empty(933 * 2, device=DEV)
    co = {n: (torch.empty(1, n, 8, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, n, 8, device=DEV)) for n in (6, 70)}
    for i in range(40):
        for t, src in zip((q, k, v), sets[i % 2]):
            t.copy_(src)
        B.gkv_prompt_attn(q, k, v, out, off, lse=lse)
        B.gkv_prompt_mass(q, k, lse, mass, off, 40)
        got = [t.clone() for t in (out, lse, mass)]
        x, n = xs[i % 4], xs[i % 4][0].shape[1]
        c.gkv_chunk_attn(0, *x, *co[n][:1], lse=co[n][1])
        c.gkv_chunk_attn(0, *xs[(i + 1) % 4], *co[76 - n][:1], lse=co[76 - n][1])
        got += [t.clone() for t in (*co[n], *co[76 - n])]
        for a, b in zip(got, (*alone[i % 2], *chunks[i % 4], *chunks[(i + 1) % 4])):
            assert torch.equal(a, b), i


def test_appends_chunks_and_reads_in_a_row():
    """Blocks close and work lists are made anew between chunks and reads that are launched behind one another: as with a wait after each call."""
    kw = dict(policy=B.POLICY_STAIRCASE, stair_tokens=(64, 128, 128, 64))
    both = []
    for waits in (True, False):
        c, oc, g = tc.caches(8, 2, 64 * 9 + 50, batch=2, seed=44, max_ctx=2048, **kw)
        new = [[t.to(DEV) for t in tc.chunk(g, 2, 6, 8, 2)] for _ in range(90)]
        kept = []
        torch.cuda.synchronize()
        for q, k, v in new:
            c.gkv_append_demote(0, k[:, :1].contiguous(), v[:, :1].contiguous())
            steps = [torch.empty_like(q), torch.empty(2, 8, 128, device=DEV)]
            if waits:
                torch.cuda.synchronize()
            c.gkv_chunk_attn(0, q, k, v, steps[0])
            if waits:
                torch.cuda.synchronize()
            c.gkv_decode_attn(0, q[:, 0].contiguous(), steps[1])
            if waits:
                torch.cuda.synchronize()
            kept.append(steps)
        torch.cuda.synchronize()
        c.gkv_bits_report(0)
        both.append(kept)
    for i, (a, b) in enumerate(zip(*both)):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), i


# ---- together ----
@pytest.mark.parametrize("turn", [5, 150])
def test_prompt_in_pieces(turn):
    """A prompt, and the next turn over the cache that holds it exactly, give the rows of one prompt of both; a decode step goes on from there."""
    n, n_q, n_kv = 64 * 7 + 21, 8, 2
    q, k, v, off = tp.make([n + turn], n_q, n_kv, seed=37)
    whole = tp.reference(q, k, v, off)
    first, l1 = tp.run(q[:n], k[:n], v[:n], np.array([0, n], dtype=np.int32))
    tp.check(first, l1, [x[:n] for x in whole], slice(0, n))
    mass = torch.empty(1, n_kv, n, device=DEV)
    B.gkv_prompt_mass(q[:n], k[:n], l1, mass, np.array([0, n], dtype=np.int32), 16)
    c = B.Cache(B.make_config(1, 1, n_q, n_kv, 128, 128, 2048, policy=B.POLICY_RD, retire_after=128, rd_budget_bpv=16.0))
    c.gkv_append_demote(0, k[:n].view(1, n, n_kv, 128), v[:n].view(1, n, n_kv, 128), token_mass=mass)
    out, lse = torch.empty(1, turn, n_q, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, turn, n_q, device=DEV)
    kt, vt = k[n:].view(1, turn, n_kv, 128), v[n:].view(1, turn, n_kv, 128)
    c.gkv_chunk_attn(0, q[n:].view(1, turn, n_q, 128), kt, vt, out, lse=lse)
    torch.cuda.synchronize()
    # (fp16 weights and rows besides the prompt's roundings: 2^-11 of the values' sum)
    o, ov, rl, mag = (x[n:] for x in whole)
    slack = 2.0 ** -16 * mag + 2.0 ** -20
    tol = (2.0 ** -8 + 2.0 ** -11) * (ov + o.abs()) * (1 + 2.0 ** -7) + 2 * slack[..., None] * ov
    assert bool(((out[0].double() - o).abs() <= tol).all()) and bool(((lse[0].double() - rl).abs() <= slack + 2.0 ** -21 * rl.abs()).all())
    for i in range(turn):
        c.gkv_append_demote(0, kt[:, i:i + 1].contiguous(), vt[:, i:i + 1].contiguous())
    dec = torch.empty(1, n_q, 128, device=DEV)
    c.gkv_decode_attn(0, q[-1:].contiguous(), dec)
    torch.cuda.synchronize()
    assert bool(((dec[0].double() - o[-1]).abs() <= tol[-1] + 2e-3).all())
    c.close()
