"""What prompt and chunk attention refuse before anything is launched, and the workspace that a prompt asks for: host arithmetic, no GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2608_23599_b200 import binding as B

P = 1 << 20                      # an address that is aligned; nothing gets as far as to read it
KEPT = []


def desc(offsets=(0, 5), n_q=8, n_kv=2, **kw):
    d = B.GkvPrompt()
    d.struct_size, d.abi_version = C.sizeof(B.GkvPrompt), B.GKV_ABI_VERSION
    off = np.asarray(offsets, dtype=np.int32)
    d.n_seqs, d.n_q_heads, d.n_kv_heads, d.head_dim, d.offsets = len(off) - 1, n_q, n_kv, 128, off.ctypes.data
    KEPT.append(off)
    for name, value in kw.items():
        setattr(d, name, value)
    return d


def attn(d, q=P, k=P, v=P, out=P, lse=None, ws=None, n=0):
    return B.load().gkv_prompt_attn(None if d is None else C.byref(d), q, k, v, out, lse, ws, n, None)


def mass(d, q=P, k=P, lse=P, m=P, n_obs=16):
    return B.load().gkv_prompt_mass(None if d is None else C.byref(d), q, k, lse, n_obs, m, None)


def room(d):
    n = C.c_size_t(0)
    return B.load().gkv_prompt_workspace_bytes(None if d is None else C.byref(d), C.byref(n)), n.value


BAD = [
    (dict(struct_size=8), B.ERR_INVALID_ARG), (dict(abi_version=B.GKV_ABI_VERSION + 1), B.ERR_INVALID_ARG), (dict(n_seqs=-1), B.ERR_INVALID_ARG),
    (dict(n_q=0), B.ERR_INVALID_ARG), (dict(n_kv=0), B.ERR_INVALID_ARG), (dict(n_q=7), B.ERR_INVALID_ARG), (dict(n_q=18), B.ERR_UNSUPPORTED),
    (dict(head_dim=64), B.ERR_UNSUPPORTED), (dict(offsets=(-1, 5)), B.ERR_INVALID_ARG), (dict(offsets=(0, 5, 4)), B.ERR_INVALID_ARG),
    (dict(q_stride=8 * 128 - 8), B.ERR_INVALID_ARG), (dict(k_stride=2 * 128 + 4), B.ERR_INVALID_ARG), (dict(v_stride=-256), B.ERR_INVALID_ARG),
    (dict(out_stride=1 << 36), B.ERR_INVALID_ARG),
]


@pytest.mark.parametrize("kw,status", BAD, ids=[next(iter(kw)) + str(i) for i, (kw, _) in enumerate(BAD)])
def test_descriptions_that_are_refused(kw, status):
    d = desc(**kw)
    assert attn(d) == status and mass(d) == status and room(d)[0] == status
    assert attn(None) == mass(None) == room(None)[0] == B.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=P + 8),
                                dict(lse=P + 2), dict(ws=P + 8, n=1 << 20)])
def test_attention_pointers(kw):
    assert attn(desc(), **kw) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(lse=None), dict(m=None), dict(q=P + 8), dict(k=P + 8), dict(lse=P + 1), dict(m=P + 2),
                                dict(n_obs=0), dict(n_obs=-3)])
def test_mass_pointers_and_observers(kw):
    assert mass(desc(), **kw) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("offsets", [(0,), (0, 0), (7, 7, 7)])
def test_nothing_to_do_needs_no_buffers(offsets):
    d = desc(offsets)
    assert attn(d, None, None, None, None) == mass(d, None, None, None, None) == B.OK and room(d) == (B.OK, 0)


def test_chunks_without_a_cache():
    n = C.c_size_t(0)
    lib = B.load()
    assert lib.gkv_chunk_attn(None, 0, P, P, P, 4, None, P, None, P, 1 << 30, None) == B.ERR_INVALID_ARG
    assert lib.gkv_chunk_workspace_bytes(None, 0, 4, C.byref(n)) == B.ERR_INVALID_ARG


def test_workspace_of_prompts():
    """Nothing where all tiles find a place at once or are alike, below 40 MB everywhere."""
    assert room(desc((0, 40))) == (B.OK, 0)
    assert room(desc((0, 4096), 32, 32)) == (B.OK, 0)
    # 100,000 tokens are 3126 tiles of up to 782 steps: eight thousand per CTA, ten times the longest
    assert room(desc((0, 100000))) == (B.OK, 0)
    for lengths in ([2500], [6000, 1, 500], [17] * 40 + [5000]):
        rc, n = room(desc(np.concatenate([[0], np.cumsum(lengths)])))
        assert rc == B.OK and 0 < n < 40 << 20, (lengths[:3], n)
    assert B.load().gkv_prompt_workspace_bytes(C.byref(desc()), None) == B.ERR_INVALID_ARG


def test_tensors_of_the_wrong_kind():
    """The binding's own checks (everything that is not a CUDA tensor ends there)."""
    q, k = torch.zeros(5, 8, 128, dtype=torch.bfloat16), torch.zeros(5, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q: a CUDA torch.bfloat16 tensor"):
        B.gkv_prompt_attn(q, k, k, q, [0, 5])
    with pytest.raises(ValueError, match="q: a CUDA"):
        B.gkv_prompt_mass(q, k, torch.zeros(5, 8), torch.zeros(10), [0, 5], 16)
    with pytest.raises(ValueError, match="q: a CUDA"):
        B.gkv_prompt_attn(None, k, k, q, [0, 5])


@pytest.mark.parametrize("bad", [[0, 5.5], np.array([0.0, 5.0]), [0, 2 ** 31], np.array([0, 2 ** 32 + 5]), ["0", "5"]])
def test_row_numbers_have_to_be_whole_numbers_of_32_bits(bad):
    with pytest.raises(ValueError, match="offsets: whole numbers"):
        B._ints(bad, "offsets")
    assert B._ints([0, 5], "x").dtype == B._ints([], "x").dtype == B._ints(torch.tensor([3]), "x").dtype == np.int32


def test_workspaces_of_four_streams_are_kept():
    spaces = {}
    for stream in (1, 2, 3, 1, 4, 5, 6):
        B._keep_space(spaces, stream, (stream, 0))
    assert list(spaces) == [1, 4, 5, 6]
