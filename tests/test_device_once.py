"""The set-up before a kernel's first launch on a device (csrc/device_once.h), compiled on its own with a stand-in for
cudaGetDevice: a set-up that has not ended, or has failed, does not count."""
import os
import subprocess
import sys
import textwrap

import pytest

from paper_2608_21614_b200 import build

PROGRAM = r"""
#include "device_once.h"
#include <cstdio>
static int device = 0;
static cudaError_t answer = cudaSuccess;
extern "C" cudaError_t CUDARTAPI cudaGetDevice(int* d) { *d = device; return answer; }
using namespace saem;
#define CHECK(c) if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; }
int main() {
    static DeviceOnce once;
    int runs = 0;
    auto good = [&] { ++runs; return cudaSuccess; };
    auto bad = [&] { ++runs; return cudaErrorInvalidValue; };
    CHECK(once_on_device(once, bad) == cudaErrorInvalidValue && runs == 1);
    CHECK(once_on_device(once, bad) == cudaErrorInvalidValue && runs == 2);          // a failure is tried again
    // another thread's call while the first one's set-up is under way: it has to set up too before it goes on
    CHECK(once_on_device(once, [&] { return once_on_device(once, good); }) == cudaSuccess && runs == 3);
    CHECK(once_on_device(once, bad) == cudaSuccess && runs == 3);                    // done
    device = 5;
    CHECK(once_on_device(once, good) == cudaSuccess && runs == 4);                   // each device for itself
    CHECK(once_on_device(once, good) == cudaSuccess && runs == 4);
    device = 64;                                                                     // beyond the table: every time
    CHECK(once_on_device(once, good) == cudaSuccess && once_on_device(once, good) == cudaSuccess && runs == 6);
    answer = cudaErrorNoDevice;
    CHECK(once_on_device(once, good) == cudaErrorNoDevice && runs == 6);
    return 0;
}
"""


def test_only_a_set_up_that_succeeded_counts(tmp_path):
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(PROGRAM)
    cuda = os.path.join(os.path.dirname(os.path.dirname(build.NVCC)), "include")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-I" + build.CSRC, "-I" + cuda, str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@pytest.mark.gpu
def test_first_calls_of_two_threads():
    """In a fresh process: each of four products and two expert layers makes its first call in two threads at once."""
    program = textwrap.dedent("""
        import threading, torch
        from paper_2608_21614_b200 import binding as B, mx
        from paper_2608_21614_b200.layer import MoELayer
        g = torch.Generator(device="cuda").manual_seed(1)
        w = mx.quantize(torch.randn(2048, 2048, generator=g, device="cuda"))
        xs = [torch.randn(m, 2048, generator=g, device="cuda") for m in (1, 300, 700, 2500)]
        q = [mx.quantize(torch.randn(128, 128, generator=g, device="cuda")) for _ in range(3)]
        layers = [MoELayer(128, 128, 4, 2, 12, ffn_path=B.SAEM_FFN_MX) for _ in range(2)]
        for layer in layers:
            for e in range(4):
                layer.load_expert_mx(0, e, e, *q)
        logits, x = torch.randn(12, 4, generator=g, device="cuda"), torch.randn(12, 128, generator=g, device="cuda").bfloat16()
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        start, out, failed = threading.Barrier(2), [None, None], []
        def work(i):
            try:
                with torch.cuda.stream(streams[i]):
                    got = []
                    for v in xs:
                        linear = mx.Linear(w, v.shape[0])
                        start.wait()
                        got.append(linear(v))
                    for T in (4, 12):
                        y = torch.empty(T, 128, device="cuda")
                        start.wait()
                        layers[i].step_fused_call(logits[:T], x[:T], T, y)
                        got.append(y)
                    streams[i].synchronize()
                    out[i] = got
            except Exception as e:
                failed.append(repr(e))
                start.abort()
        threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
        [t.start() for t in threads]
        [t.join() for t in threads]
        assert not failed, failed
        assert all(torch.equal(a, b) for a, b in zip(*out))
        print("same")
    """)
    r = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300, cwd=os.path.dirname(os.path.dirname(__file__)))
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
