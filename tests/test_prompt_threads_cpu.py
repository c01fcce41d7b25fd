"""Prompt calls of several host threads, without a GPU: what the extension holds while the interpreter is unlocked, and in which order launches are made."""
import ctypes as C
import importlib.machinery
import importlib.util
import shutil
import weakref

import numpy as np
import pytest

from paper_2608_23599_b200 import binding as B
from paper_2608_23599_b200 import build as _build


class Rows:
    """What the extension asks of a tensor."""
    dtype = "bf16"

    def __init__(self, *shape):
        self.shape = shape

    def get_device(self):
        return 0

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def extension(tmp_path):
    """A second copy of the extension, to be bound to fakes."""
    B.load()
    path = shutil.copy(_build.CALL_LIB, tmp_path)
    spec = importlib.util.spec_from_file_location("_gkv_call", path, loader=importlib.machinery.ExtensionFileLoader("_gkv_call", path))
    return importlib.util.module_from_spec(spec)


def test_a_streams_workspace_is_held_until_the_launches_are_made(extension):
    """Another thread replaces the stream's workspace while this one is inside the library."""
    class Memory:
        pass

    spaces, seen = {}, []
    memory = Memory()
    alive = weakref.ref(memory)
    spaces[64 * 0x77] = (1 << 24, 4096, memory)
    del memory

    def bytes_needed(_, need):
        need[0] = 4096
        return 0

    def attn(d, q, k, v, out, lse, ws, n, st):
        spaces.clear()
        seen.append((ws, n, alive() is not None))
        return 0

    vp = C.c_void_p
    fakes = [C.CFUNCTYPE(C.c_int, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp)(attn), C.CFUNCTYPE(C.c_int, vp, C.POINTER(C.c_size_t))(bytes_needed)]
    a, b = (C.cast(f, vp).value for f in fakes)
    extension.bind_rows(a, b, 0, 0, Rows, Rows.dtype, "f32", lambda: 0, lambda d: 0x77, lambda: False)
    q, k, off = Rows(5, 8, 128), Rows(5, 2, 128), np.array([0, 5], dtype=np.int32)
    assert extension.prompt_attn(q, k, k, q, off, None, 0.0, spaces) == 0
    assert seen == [(1 << 24, 4096, True)]
    assert alive() is None                           # (and given back behind them)
