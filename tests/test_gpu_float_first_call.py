"""Calls from threads in every state: the first ones of a process, from several threads at once, with another context current or none."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


def run(program):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([os.path.dirname(HERE), HERE, os.environ.get("PYTHONPATH", "")]))
    done = subprocess.run([sys.executable, "-c", program], env=env, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "same" in done.stdout, done.stderr[-2000:]


def test_first_calls_from_eight_threads_at_once():
    run("""
import threading
import torch
import test_gpu_float_ops as ops
from paper_2011_10680_b200 import binding
hq = binding.Handle(0)
states = [ops.block_state(70, 702) for _ in range(4)] + [ops.block_state(5, 703) for _ in range(4)]
torch.cuda.synchronize()
start = threading.Barrier(8)
def work(t):
    with torch.cuda.stream(torch.cuda.Stream()):
        start.wait()
        ops.block(hq, t)
        torch.cuda.current_stream().synchronize()
threads = [threading.Thread(target=work, args=(t,)) for t in states]
[t.start() for t in threads]
[t.join() for t in threads]
hq.sync()
for t, first in [(t, states[0]) for t in states[1:4]] + [(t, states[4]) for t in states[5:]]:
    assert all(torch.equal(t[k].view(torch.uint8), first[k].view(torch.uint8)) for k in ops.RESULTS)
again = ops.block_state(70, 702)
ops.block(hq, again)
hq.sync()
assert all(torch.equal(again[k].view(torch.uint8), states[0][k].view(torch.uint8)) for k in ops.RESULTS)
print("same")
""")


def test_the_threads_context_stays_current():
    """A thread with a context of its own on the same device, and one with none: calls run in the handle's and leave the thread's."""
    run("""
import ctypes as C
import threading
import torch
import test_gpu_float_ops as ops
from paper_2011_10680_b200 import binding
cuda = C.CDLL("libcuda.so.1")
def check(code):
    assert code == 0, code
def current():
    c = C.c_void_p()
    check(cuda.cuCtxGetCurrent(C.byref(c)))
    return c.value
hq = binding.Handle(0)
want = ops.block_state(40, 702)
ops.block(hq, want)
hq.sync()
states = [ops.block_state(40, 702) for _ in range(3)]
torch.cuda.synchronize()
seen = []
def own_context():
    mine = C.c_void_p()
    check(cuda.cuCtxCreate_v2(C.byref(mine), 0, 0))
    ops.block(hq, states[0])
    seen.append(current() == mine.value)
    other = C.c_void_p()                       # and another one, after calls have been made from this thread
    check(cuda.cuCtxCreate_v2(C.byref(other), 0, 0))
    ops.block(hq, states[1])
    seen.append(current() == other.value)
    check(cuda.cuCtxDestroy_v2(other))
    check(cuda.cuCtxDestroy_v2(mine))
def no_context():
    check(cuda.cuCtxSetCurrent(None))
    ops.block(hq, states[2])
    seen.append(current() is None)
for work in (own_context, no_context):
    thread = threading.Thread(target=work)
    thread.start()
    thread.join()
torch.cuda.synchronize()
hq.sync()
assert seen == [True, True, True], seen
for t in states:
    assert all(torch.equal(t[k].view(torch.uint8), want[k].view(torch.uint8)) for k in ops.RESULTS)
print("same")
""")
