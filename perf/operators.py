"""Timed cases of what stands around single-token decode on the graded KV cache: the prompt, and chunks of new tokens.

Three operators, each one pass of one layer:

  prompt  causal attention of packed prompts over their own exact keys and values, with the log-sum-exp per row
          (`gkv_prompt_attn`): what produces the activations behind the rows that a bulk ingest takes
  mass    the attention mass that each prompt token gets from the newest queries of its sequence, averaged over them and
          over the query heads of a KV head (`gkv_prompt_mass`): the token masses that the rate-distortion policy and the
          exact residual rows of a bulk ingest are chosen by
  chunk   attention of several new tokens per sequence over the graded cache and, causally, over one another
          (`Cache.gkv_chunk_attn`): verification of drafted tokens, and the next turn of a conversation

`own` chooses between the plain form (elementary torch operations in 32 bits) and the framework's calls.
"""
import math

import numpy as np
import torch

own = False

D, BLOCK, GROUP = 128, 64, 32
DEV = "cuda"


# ---- cases ---------------------------------------------------------------------------------------
def _prompt(name, n_q, n_kv, lengths, fused=False):
    c = dict(kind="prompt", n_q=n_q, n_kv=n_kv, lengths=" ".join(str(n) for n in lengths), fused=fused)
    return dict(c, name=name) if name else c


def _mass(name, n_q, n_kv, lengths, n_obs):
    c = dict(kind="mass", n_q=n_q, n_kv=n_kv, lengths=" ".join(str(n) for n in lengths), n_obs=n_obs)
    return dict(c, name=name) if name else c


def _chunk(name, batch, n_q, n_kv, ctx, n_new, *, w16=0, w8=0, w4=0, w2=0, mixed=False, ragged=False):
    c = dict(kind="chunk", batch=batch, n_q=n_q, n_kv=n_kv, ctx=ctx, n_new=n_new, w16=w16, w8=w8, w4=w4, w2=w2, mixed=mixed, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # three chat messages that arrive together on a small model, one of them a single token: all latency
        _prompt("prompt_tiny", 8, 2, [1, 75, 33]),
        # a batch of requests of very different lengths, as a serving scheduler packs them, rows inside a fused q|k|v projection
        _prompt("prompt_ragged_8b", 32, 8, [1023, 17, 2048, 333, 0, 640, 129, 1501], fused=True),
        # one prompt of ordinary length with a KV head per query head
        _prompt("prompt_mha_4k", 8, 8, [4097]),
        # a long prompt with eight query heads per KV head
        _prompt("prompt_gqa8_16k", 16, 2, [16384]),
        # masses of a short prompt, before its ingest
        _mass("mass_2k", 8, 2, [2072], 16),
        # masses of a batch of long prompts: the keys are read once
        _mass("mass_8b_32k", 32, 8, [32768, 20001, 4097], 16),
        # a wider observation window over a long prompt
        _mass("mass_wide_16k", 16, 2, [16384], 64),
        # four drafted tokens on a short conversation: all latency
        _chunk("verify_1k", 1, 8, 2, 1000, 4, w16=256, w8=256, w4=256, w2=128),
        # five drafted tokens per sequence of a batch over long contexts on every rung of the ladder
        _chunk("verify_8b_32k", 8, 32, 8, 32757, 5, w16=1024, w8=4096, w4=16384, w2=8192),
        # sixteen drafted tokens over a plan that differs from block to block and from head to head
        _chunk("verify_mixed_8k", 2, 32, 8, 8200, 16, mixed=True),
        # the next turn of two conversations, messages of different lengths
        _chunk("turn_8k", 2, 32, 8, 8191, 300, w16=512, w8=2048, w4=4096, ragged=True),
        # a long document behind a long cached context
        _chunk("turn_long", 1, 16, 2, 32768, 2000, w16=1024, w8=4096, w4=16384, w2=8192),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(8, 2), (16, 2), (32, 8), (12, 4), (14, 2), (8, 8), (10, 2), (4, 1)]


def draw(rng):
    n_q, n_kv = rng.choice(HEADS)
    kind = rng.choice(["prompt", "mass", "chunk", "chunk"])
    if kind == "prompt":
        top = int(math.sqrt(16.0 * 16000 * 16000 / n_q))
        total = _log_int(rng, 16, min(top, 16000))
        n = rng.choice([1, 1, 2, 3, 5, 9])
        cuts = sorted(rng.randint(0, total) for _ in range(n - 1))
        lengths = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        return _prompt("", n_q, n_kv, lengths, fused=rng.random() < 0.3)
    if kind == "mass":
        lengths = [_log_int(rng, 100, 30000) for _ in range(rng.choice([1, 1, 2, 4]))]
        return _mass("", n_q, n_kv, lengths, rng.choice([1, 8, 16, 32, 50, 64]))
    batch = rng.choice([1, 1, 2, 3, 5])
    ctx = _log_int(rng, 600, 30000)
    n_new = _log_int(rng, 1, max(2, min(1500, int(1.0e9 / (batch * n_q * ctx)))))
    parts = [rng.uniform(0.03, 0.2), rng.uniform(0.05, 0.4), rng.uniform(0.1, 0.5), rng.uniform(0.0, 0.3)]
    w = [max(1, int(p * ctx / BLOCK)) * BLOCK for p in parts]
    return _chunk("", batch, n_q, n_kv, ctx, n_new, w16=w[0], w8=w[1], w4=w[2], w2=w[3], mixed=rng.random() < 0.3, ragged=batch > 1 and rng.random() < 0.5)


# ---- inputs --------------------------------------------------------------------------------------
def _lengths(case):
    return [int(n) for n in case["lengths"].split()]


def _levels(case, gen):
    """Rung of every closed block, oldest first: the staircase by age, or one drawn per block and stream."""
    b, h, nb = case["batch"], case["n_kv"], case["ctx"] // BLOCK
    if case["mixed"]:
        pick = torch.tensor([16, 8, 4, 4, 2, 1], dtype=torch.int8, device=DEV)
        return pick[torch.randint(0, 6, (b, h, nb), generator=gen, device=DEV)]
    age = torch.arange(nb - 1, -1, -1, device=DEV) * BLOCK          # tokens of closed blocks that are newer
    edges = torch.tensor([case["w16"], case["w8"], case["w4"], case["w2"]], device=DEV).cumsum(0)
    rung = torch.tensor([16, 8, 4, 2, 1], dtype=torch.int8, device=DEV)[torch.bucketize(age, edges, right=True)]
    return rung.expand(b, h, nb).contiguous()


def _codes(x, qmax):
    """Asymmetric min/max codes of groups along the last dimension: (codes, scale, zero point)."""
    lo, hi = x.amin(-1), x.amax(-1)
    s, z = ((hi - lo) / qmax).half(), lo.half()
    s32, z32 = s.float(), z.float()
    inv = torch.where(s32 > 0, 1.0 / s32, torch.zeros_like(s32))
    code = ((x - z32[..., None]) * inv[..., None]).round_().clamp_(min=0.0)
    return torch.minimum(code, qmax[..., None].expand_as(code)).to(torch.uint8), s, z


def _centroid(x):
    acc = torch.zeros_like(x[..., 0, :])
    for t in range(BLOCK):
        acc = acc + x[..., t, :]
    return (acc * (1.0 / BLOCK)).bfloat16()


def _graded(rows, levels, keys):
    """The stored form of [b, t, h, 128] rows on their rungs: codes [b, h, block, 64, 128], scales and zero points, centroids."""
    b, h, nb = levels.shape
    x = rows[:, : nb * BLOCK].float().view(b, nb, BLOCK, h, D).permute(0, 3, 1, 2, 4)
    bits = torch.where((levels == 16) | (levels == 1), 8, levels.long())
    qmax = (2.0 ** bits.float()) - 1.0
    if keys:      # 32 tokens x 1 channel
        g = x.reshape(b, h, nb, 2, GROUP, D).transpose(-1, -2)
        code, s, z = _codes(g, qmax[..., None, None].expand(b, h, nb, 2, D))
        code = code.transpose(-1, -2).reshape(b, h, nb, BLOCK, D)
    else:         # 1 token x 32 channels
        g = x.reshape(b, h, nb, BLOCK, D // GROUP, GROUP)
        code, s, z = _codes(g, qmax[..., None, None].expand(b, h, nb, BLOCK, D // GROUP))
        code = code.reshape(b, h, nb, BLOCK, D)
    return dict(code=code.contiguous(), s=s.contiguous(), z=z.contiguous(), mean=_centroid(x), rows=rows)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    n_q, n_kv = case["n_q"], case["n_kv"]
    # a few key channels of every head are much larger than the others, as in trained models
    gain = torch.ones((n_kv, D), device=DEV)
    for h in range(n_kv):
        gain[h, torch.randperm(D, generator=gen, device=DEV)[:4]] = 8.0
    s = dict(kind=case["kind"], n_q=n_q, n_kv=n_kv, scale=1.0 / math.sqrt(D))
    if case["kind"] in ("prompt", "mass"):
        lengths = _lengths(case)
        s["offsets"] = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        s["offsets_dev"] = torch.from_numpy(s["offsets"]).to(DEV)
        t = int(s["offsets"][-1])
        q, k, v = randn(t, n_q, D).bfloat16(), (randn(t, n_kv, D) * gain).bfloat16(), randn(t, n_kv, D).bfloat16()
        if case["kind"] == "prompt":
            if case["fused"]:      # slices of one projection's output
                qkv = torch.cat([q, k, v], dim=1)
                q, k, v = qkv[:, :n_q], qkv[:, n_q : n_q + n_kv], qkv[:, n_q + n_kv :]
            s.update(q=q, k=k, v=v, out=torch.empty((t, n_q, D), dtype=torch.bfloat16, device=DEV), lse=torch.empty((t, n_q), device=DEV))
            return s
        # the log-sum-exp that the prompt's attention left; only the observing rows matter here
        lse = torch.zeros((t, n_q), device=DEV)
        for a, b in zip(s["offsets"][:-1].tolist(), s["offsets"][1:].tolist()):
            o = min(case["n_obs"], b - a)
            kk = k[a:b].double()
            for h in range(n_q if o else 0):
                x = (q[b - o : b, h].double() @ kk[:, h // (n_q // n_kv)].t()) * s["scale"]
                x += torch.full((o, b - a), -math.inf, dtype=x.dtype, device=DEV).triu_(b - a - o + 1)
                lse[b - o : b, h] = torch.logsumexp(x, -1).float()
        s.update(q=q, k=k, lse=lse, n_obs=case["n_obs"], mass=torch.empty(t * n_kv, device=DEV))
        return s
    b, t, n = case["batch"], case["ctx"], case["n_new"]
    levels = _levels(case, gen)
    k = (randn(b, t, n_kv, D) * gain).bfloat16()
    v = randn(b, t, n_kv, D).bfloat16()
    lengths = [n] * b
    if case["ragged"]:
        lengths = [max(0, n - i * (n // b + 1)) if i % 2 else n - i for i in range(b)]
        lengths = [max(0, x) for x in lengths]
    s.update(levels=levels, q=randn(b, n, n_q, D).bfloat16(), k_new=(randn(b, n, n_kv, D) * gain).bfloat16(), v_new=randn(b, n, n_kv, D).bfloat16(),
             lengths=np.array(lengths, dtype=np.int32), lengths_dev=torch.tensor(lengths, device=DEV),
             out=torch.zeros((b, n, n_q, D), dtype=torch.bfloat16, device=DEV), lse=torch.zeros((b, n, n_q), device=DEV))
    if own:      # the handle that a serving program keeps
        from paper_2608_23599_b200 import binding as B
        s["cache"] = B.Cache(B.make_config(1, b, n_q, n_kv, D, D, t + 64, policy=B.POLICY_EXTERNAL))
        s["cache"].gkv_append_demote(0, k, v, level_plan=levels.cpu().numpy())
    else:
        s["k"], s["v"] = _graded(k, levels, True), _graded(v, levels, False)
    return s


# ---- one pass ------------------------------------------------------------------------------------
def _plain_prompt(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    t, n_q, n_kv = q.shape[0], s["n_q"], s["n_kv"]
    g = n_q // n_kv
    pos = torch.arange(t, device=DEV)
    seq = torch.bucketize(pos, s["offsets_dev"][1:], right=True)
    hidden = (seq[:, None] != seq[None, :]) | (pos[None, :] > pos[:, None])
    x = torch.matmul(q.view(t, n_kv, g, D).permute(1, 2, 0, 3), k.permute(1, 2, 0)[:, None]).mul_(s["scale"])      # [n_kv, g, t, t]
    x.masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v.permute(1, 0, 2)[:, None]) / total
    lse = (top + total.log())[..., 0]
    return o.permute(2, 0, 1, 3).reshape(t, n_q, D).bfloat16(), lse.permute(2, 0, 1).reshape(t, n_q)


def _plain_mass(s):
    q, k, off = s["q"], s["k"].float(), s["offsets_dev"]
    t, n_q, n_kv, n_obs = q.shape[0], s["n_q"], s["n_kv"], s["n_obs"]
    g, n = n_q // n_kv, off.numel() - 1
    length = (off[1:] - off[:-1]).long()
    # the observing rows of every sequence: [n, n_obs], the newest last; rows before a short sequence's start count nothing
    row = off[1:, None].long() - n_obs + torch.arange(n_obs, device=DEV)
    real = row >= off[:-1, None]
    row = row.clamp(0, t - 1)
    qo, lo = q[row].float(), s["lse"][row]                                # [n, n_obs, n_q, (D)]
    pos = torch.arange(t, device=DEV)
    seq = torch.bucketize(pos, off[1:], right=True)
    x = torch.matmul(qo.view(n, n_obs, n_kv, g, D).permute(2, 0, 1, 3, 4).reshape(n_kv, n * n_obs * g, D), k.permute(1, 2, 0)).mul_(s["scale"])
    x = x.view(n_kv, n, n_obs, g, t) - lo.view(n, n_obs, n_kv, g).permute(2, 0, 1, 3)[..., None]
    seen = real[:, :, None] & (seq[None, None] == torch.arange(n, device=DEV)[:, None, None]) & (pos <= row[:, :, None])      # [n, n_obs, t]
    x = torch.where(seen[None, :, :, None], x.exp(), torch.zeros((), device=DEV))
    m = x.sum((1, 2, 3)) / (g * length.clamp(max=n_obs)).float()[seq]     # [n_kv, t]
    # laid out sequence after sequence, [n_kv][length] each
    place = off[seq].long() * n_kv + (pos - off[seq])
    mass = torch.empty(n_kv * t, device=DEV)
    mass[place + torch.arange(n_kv, device=DEV)[:, None] * length[seq]] = m
    return mass


def _rows(x, levels, keys):
    """Stored blocks as 32-bit rows [b, h, tokens, 128], the exact partial block behind them."""
    b, h, nb = levels.shape
    c, s, z = x["code"].float(), x["s"].float(), x["z"].float()
    if keys:
        s, z = s.repeat_interleave(GROUP, 3), z.repeat_interleave(GROUP, 3)
    else:
        s, z = s.repeat_interleave(GROUP, 4), z.repeat_interleave(GROUP, 4)
    r = torch.addcmul(z, c, s)
    exact = x["rows"].float().transpose(1, 2)
    lv = levels[..., None, None]
    r = torch.where(lv == 16, exact[:, :, : nb * BLOCK].reshape(b, h, nb, BLOCK, D), torch.where(lv == 1, x["mean"].float()[..., None, :], r))
    return torch.cat([r.view(b, h, nb * BLOCK, D), exact[:, :, nb * BLOCK :]], dim=2)


def _plain_chunk(s):
    q, levels = s["q"].float(), s["levels"]
    b, n, n_q, _ = q.shape
    n_kv = s["n_kv"]
    g = n_q // n_kv
    k = torch.cat([_rows(s["k"], levels, True), s["k_new"].float().transpose(1, 2)], dim=2)
    v = torch.cat([_rows(s["v"], levels, False), s["v_new"].float().transpose(1, 2)], dim=2)
    t = k.shape[2] - n
    x = torch.matmul(q.view(b, n, n_kv, g, D).permute(0, 2, 3, 1, 4).reshape(b, n_kv, g * n, D), k.transpose(-1, -2)).mul_(s["scale"])
    x = x.view(b, n_kv, g, n, t + n)
    x[..., t:].masked_fill_(torch.ones((n, n), dtype=torch.bool, device=DEV).triu_(1), -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(b, n_kv, g * n, t + n), v).view(b, n_kv, g, n, D) / total
    real = torch.arange(n, device=DEV) < s["lengths_dev"][:, None]
    out = torch.where(real[:, :, None, None], o.permute(0, 3, 1, 2, 4).reshape(b, n, n_q, D), torch.zeros((), device=DEV))
    lse = torch.where(real[:, :, None], (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(b, n, n_q), torch.zeros((), device=DEV))
    return out.bfloat16(), lse


def run(s):
    if own:
        if s["kind"] == "prompt":
            from paper_2608_23599_b200 import binding as B
            B.gkv_prompt_attn(s["q"], s["k"], s["v"], s["out"], s["offsets"], lse=s["lse"])
            return s["out"], s["lse"]
        if s["kind"] == "mass":
            from paper_2608_23599_b200 import binding as B
            B.gkv_prompt_mass(s["q"], s["k"], s["lse"], s["mass"], s["offsets"], s["n_obs"])
            return s["mass"]
        s["cache"].gkv_chunk_attn(0, s["q"], s["k_new"], s["v_new"], s["out"], lse=s["lse"], lengths=s["lengths"])
        return s["out"], s["lse"]
    return {"prompt": _plain_prompt, "mass": _plain_mass, "chunk": _plain_chunk}[s["kind"]](s)


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    n_q, n_kv = case["n_q"], case["n_kv"]
    if case["kind"] == "prompt":
        t = sum(_lengths(case))
        pairs = sum(n * (n + 1) // 2 for n in _lengths(case))
        return dict(bytes=t * (2 * n_q + 2 * n_kv) * D * 2 + t * n_q * 4, flops=4 * D * n_q * pairs)
    if case["kind"] == "mass":
        o = [min(case["n_obs"], n) for n in _lengths(case)]
        t = sum(_lengths(case))
        pairs = sum(a * n - a * (a - 1) // 2 for a, n in zip(o, _lengths(case)))
        return dict(bytes=t * n_kv * (D * 2 + 4) + sum(o) * n_q * (D * 2 + 4), flops=2 * D * n_q * pairs)
    b, t, n = case["batch"], case["ctx"], case["n_new"]
    nb = t // BLOCK
    per_block = {16: 32768, 8: 18432, 4: 10240, 2: 6144, 1: 512}
    if case["mixed"]:
        cache = nb * sum(per_block[x] for x in (16, 8, 4, 4, 2, 1)) / 6
        keys = nb * (5 * BLOCK + 1) / 6
    else:
        cache, keys, left = 0, 0, nb
        for lv, w in ((16, case["w16"]), (8, case["w8"]), (4, case["w4"]), (2, case["w2"]), (1, t)):
            m = min(left, w // BLOCK if lv > 1 else left)
            cache, keys, left = cache + m * per_block[lv], keys + m * (BLOCK if lv > 1 else 1), left - m
    tail = t % BLOCK
    ragged = [max(0, n - i * (n // b + 1)) if i % 2 else max(0, n - i) for i in range(b)] if case["ragged"] else [n] * b
    rows = sum(ragged)
    pairs = sum(m * (keys + tail) + m * (m + 1) // 2 for m in ragged)
    seen = sum(1 for m in ragged if m)
    return dict(bytes=seen * n_kv * (cache + tail * 512) + rows * (2 * n_q + 2 * n_kv) * D * 2 + rows * n_q * 4, flops=4 * D * n_q * pairs)


# ---- the definition in 64 bits -------------------------------------------------------------------
def _attend(q, k, v, scale, first):
    """Softmax attention of rows q [m, D] over k, v [n, D]; row i sees the keys up to first + i."""
    x = (q @ k.T) * scale
    m, n = x.shape
    x = torch.where(torch.arange(n, device=DEV)[None] <= first + torch.arange(m, device=DEV)[:, None], x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, dim=1)
    return torch.exp(x - lse[:, None]) @ v, lse


def _decode_block(x, i, h, j, level, keys):
    """Block j of stream (i, h) as 64-bit rows, from what is stored."""
    if level == 16:
        return x["rows"][i, j * BLOCK : (j + 1) * BLOCK, h].double()
    if level == 1:
        return x["mean"][i, h, j].double().expand(BLOCK, D)
    c, s, z = x["code"][i, h, j].double(), x["s"][i, h, j].double(), x["z"][i, h, j].double()
    if keys:
        c = c.view(2, GROUP, D)
        return (c * s[:, None] + z[:, None]).view(BLOCK, D)
    return (c.view(BLOCK, D // GROUP, GROUP) * s[..., None] + z[..., None]).view(BLOCK, D)


def exact(case, seed):
    global own
    asked, own = own, False      # the stored form of the cache in plain tensors
    s = prepare(case, seed)
    own = asked
    n_q, g = s["n_q"], s["n_q"] // s["n_kv"]
    scale = 1.0 / math.sqrt(128.0)
    if s["kind"] == "chunk":
        levels = s["levels"].cpu().tolist()
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
        lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
        for i, m in enumerate(s["lengths"].tolist()):
            for h in range(s["n_kv"] if m else 0):
                rows = []
                for x, new, keys in ((s["k"], s["k_new"], True), (s["v"], s["v_new"], False)):
                    blocks = [_decode_block(x, i, h, j, lv, keys) for j, lv in enumerate(levels[i][h])]
                    rows.append(torch.cat(blocks + [x["rows"][i, len(blocks) * BLOCK :, h].double(), new[i, :m, h].double()]))
                for a in range(h * g, (h + 1) * g):
                    out[i, :m, a], lse[i, :m, a] = _attend(s["q"][i, :m, a].double(), rows[0], rows[1], scale, case["ctx"])
        return out, lse
    t = int(s["offsets"][-1])
    if s["kind"] == "prompt":
        out, lse = torch.zeros((t, n_q, D), dtype=torch.float64, device=DEV), torch.zeros((t, n_q), dtype=torch.float64, device=DEV)
    else:
        out = torch.zeros(t * s["n_kv"], dtype=torch.float64, device=DEV)
    start = 0
    for length in _lengths(case):
        end = start + length
        for a in range(n_q if length else 0):
            k = s["k"][start:end, a // g].double()
            if s["kind"] == "prompt":
                v = s["v"][start:end, a // g].double()
                for r in range(start, end, 4096):
                    e = min(end, r + 4096)
                    out[r:e, a], lse[r:e, a] = _attend(s["q"][r:e, a].double(), k[: e - start], v[: e - start], scale, r - start)
            else:
                o = min(case["n_obs"], length)
                w = torch.exp((s["q"][end - o : end, a].double() @ k.T) * scale - s["lse"][end - o : end, a].double()[:, None]).tril_(length - o)
                at = start * s["n_kv"] + (a // g) * length
                out[at : at + length] += w.sum(0) / (o * g)
        start = end
    return (out, lse) if s["kind"] == "prompt" else out
