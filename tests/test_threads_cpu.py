"""The binding called from two threads, each on a stream of its own, against a
library that only notes on which stream its entries run (no GPU): the stream is
one for the whole process, so setting it and making the call belong together."""
import threading
import types

import pytest
import torch

from paper_1810_09958_gb300 import isam

F32, BF16, I32, U8 = torch.float32, torch.bfloat16, torch.int32, torch.uint8


class Tensor:
    """What the binding asks of a contiguous tensor on device 0."""

    is_cuda = True

    def __init__(self, n, dtype):
        self.n, self.dtype = n, dtype

    def get_device(self):
        return 0

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


class Library:
    """Threads that both get as far as setting the stream go on together."""

    def __init__(self):
        self.stream, self.ran, self.both = None, {}, threading.Barrier(2)

    def isam_set_stream(self, stream):
        self.stream = stream
        try:
            self.both.wait(0.3)
        except threading.BrokenBarrierError:
            pass
        return 0

    def isam_glu_backward_workspace(self, T, D, F, out):
        out._obj.value = 64
        return 0

    def __getattr__(self, name):
        def entry(*args):
            self.ran[threading.current_thread().name] = self.stream
            return 0
        return entry


def b(n):
    return Tensor(n, BF16)


def f(n):
    return Tensor(n, F32)


def u(n):
    return Tensor(n, U8)


CALLS = {
    "gemm": lambda: isam.gemm(8, 8, 8, 0, 0, 1.0, b(64), b(64), 0.0, f(64)),
    "gemm_fp8": lambda: isam.gemm_fp8(8, 8, 16, 1.0, u(128), u(128), 0.0, f(64)),
    "gemm_mxfp8": lambda: isam.gemm_mxfp8(8, 8, 32, 1.0, u(256), u(32), u(256), u(32), 0.0, f(64)),
    "gemm_grouped": lambda: isam.gemm_grouped([(8, 8, 8, 0, 0, 1.0, b(64), b(64), 0.0, f(64))]),
    "grouped_fp8": lambda: isam.GroupedGemmFp8([(8, 8, 16, 1.0, u(128), u(128), 0.0, f(64))])(),
    "grouped_mxfp8": lambda: isam.GroupedGemmMxfp8([(8, 8, 32, 1.0, u(256), u(32), u(256), u(32), 0.0, f(64))])(),
    "gru_forward": lambda: isam.gru_forward(2, 1, 8, b(16), b(192), b(192), f(48), None, f(16)),
    "gru_forward_stack": lambda: isam.gru_forward_stack(1, 2, 1, 8, b(16), b(192), b(192), f(48), None, f(16)),
    "dwsep_conv": lambda: isam.dwsep_conv(1, 4, 4, 16, 16, b(256), b(144), b(256), f(256)),
    "depthwise_conv3x3": lambda: isam.depthwise_conv3x3(1, 4, 4, 16, b(256), b(144), b(256)),
    "glr_forward": lambda: isam.glr_forward(2, 1, 8, f(32), None, None, b(16)),
    "glr_backward": lambda: isam.glr_backward(2, 1, 8, f(32), None, None, b(16), b(16), None, f(32)),
    "glr_step": lambda: isam.glr_step(1, 8, 1, f(16), None, f(8), f(8), b(8)),
    "glu_forward": lambda: isam.glu_forward(2, 8, 8, "silu", b(16), b(128), b(16)),
    "glu_backward": lambda: isam.glu_backward(2, 8, 8, "silu", b(16), b(128), b(16), b(16), b(128), u(64)),
    "glu_backward_own_workspace": lambda: isam.glu_backward(2, 8, 8, "silu", b(16), b(128), b(16), b(16), b(128)),
    "w4_pack": lambda: isam.w4_pack(16, 128, 128, u(1024), b(16), u(1024), b(16)),
    "gemv_w4": lambda: isam.gemv_w4(1, 16, 128, 128, b(128), u(1024), b(16), f(16)),
}


@pytest.mark.parametrize("name", CALLS)
def test_each_thread_runs_on_its_own_stream(name, monkeypatch):
    lib, mine, workspaces = Library(), threading.local(), {}

    def alloc(size, stream):
        workspaces[threading.current_thread().name] = stream
        return 8192

    allocator = types.SimpleNamespace(_cuda_cudaCachingAllocator_raw_alloc=alloc,
                                      _cuda_cudaCachingAllocator_raw_delete=lambda at: None)
    monkeypatch.setattr(isam, "_torch", types.SimpleNamespace(float32=F32, bfloat16=BF16, int32=I32, uint8=U8, _C=allocator))
    monkeypatch.setattr(isam, "_kinds", {F32: 0, BF16: 1})
    monkeypatch.setattr(isam, "_lib", lib)
    monkeypatch.setattr(isam, "_current_device", lambda: 0)
    monkeypatch.setattr(isam, "_raw_stream", lambda device: mine.stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    failed = []

    def work(stream):
        mine.stream = stream
        try:
            CALLS[name]()
        except Exception as e:  # (an exception in a thread does not fail a test by itself)
            failed.append(e)

    threads = {s: threading.Thread(target=work, args=(s,), name=f"stream {s}") for s in (1, 2)}
    for t in threads.values():
        t.start()
    for t in threads.values():
        t.join(30)
    assert not failed, failed
    assert lib.ran == {t.name: s for s, t in threads.items()}
    if name == "glu_backward_own_workspace":
        assert workspaces == lib.ran
