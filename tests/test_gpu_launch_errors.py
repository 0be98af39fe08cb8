"""What a call leaves behind when a launch fails."""
import ctypes

import pytest

from paper_2406_06385_gb300 import lrqat as LQ

from gpu_util import torch

pytestmark = pytest.mark.gpu


def _ints(v):
    t = torch()
    return t.tensor(v, dtype=t.int32, device="cuda")


def _runtime():
    """The CUDA runtime that torch has loaded."""
    torch().cuda.init()
    with open("/proc/self/maps") as f:
        paths = {line.split()[-1] for line in f if "/libcudart" in line}
    if not paths:
        pytest.skip("torch has no shared CUDA runtime")
    return ctypes.CDLL(sorted(paths)[0])


class Small:
    """A truncation and an attention call of a few tokens."""

    def __init__(self):
        t = torch()
        self.table, self.ids = t.arange(8, device="cuda").int().view(2, 4), _ints([0] * 16)
        self.blocks = LQ.KVBlocks.of(self.table, self.ids, 16, 0)
        self.lens, self.keep, self.free = _ints([40, 20]), _ints([10, 20]), _ints([0])
        self.room = t.empty(LQ.kv_blocks_workspace_bytes(self.blocks), dtype=t.uint8, device="cuda")
        codes = t.zeros(8, 1, 16, 64, dtype=t.int8, device="cuda")
        scale = t.ones(8, 1, device="cuda")
        self.cache = LQ.KVCache.of(codes, codes, scale, scale)
        self.batch = LQ.KVBatch.of(_ints([40, 20]), _ints([0, 1, 2]), self.table, 2, 1, 64)
        self.q = t.ones(2, 1, 64, device="cuda").bfloat16()
        self.out = t.empty_like(self.q)

    def attend(self, **kw):
        LQ.kv_attn_sinks(self.cache, self.batch, self.q, 0.1, 0, 0, self.out, None, **kw)

    def shorten(self):
        out, free = _ints([0, 0]), _ints([0])
        LQ.kv_truncate(self.blocks, self.lens, self.keep, self.free, out, free, self.room)
        assert out.tolist() == [10, 20] and free.tolist() == [2]


def test_a_failed_launch_does_not_fail_the_next_call():
    """The runtime refuses a launch into the legacy stream while a blocking stream is being captured (and would refuse it
    for any other reason alike); the call behind it is in order."""
    runtime, small, stream, graph = _runtime(), Small(), ctypes.c_void_p(), ctypes.c_void_p()
    small.attend()
    small.shorten()
    assert runtime.cudaStreamCreate(ctypes.byref(stream)) == 0
    assert runtime.cudaStreamBeginCapture(stream, 2) == 0            # relaxed: nothing else is refused meanwhile
    try:
        with pytest.raises(LQ.LrqatError) as e:
            small.attend(stream=0)
    finally:
        runtime.cudaStreamEndCapture(stream, ctypes.byref(graph))
        if graph.value:
            runtime.cudaGraphDestroy(graph)
        runtime.cudaStreamDestroy(stream)
        runtime.cudaGetLastError()                                   # torch's runtime keeps an error of its own
    assert e.value.status == -5
    small.shorten()
    small.attend()
    LQ.get_device_status()
