"""The operators' calls run with their tensors' device current, shown on the CPU
with a device type of the test's own that counts as two devices."""
import os
import subprocess
import sys
import sysconfig

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DEVICES = r"""
#include <torch/csrc/Dtype.h>
#include <torch/csrc/utils/pybind.h>
#include <ATen/ATen.h>
#include <c10/core/impl/FakeGuardImpl.h>

// two devices with nothing behind them; which one is current is all there is
using Fake = c10::impl::FakeGuardImpl<c10::DeviceType::PrivateUse1>;
C10_REGISTER_GUARD_IMPL(PrivateUse1, Fake)

at::Tensor empty(std::vector<int64_t> shape, py::object dtype, int index) {
  const c10::Device dev(c10::DeviceType::PrivateUse1, index);
  c10::Storage none(c10::Storage::use_byte_size_t(), 1 << 20, c10::DataPtr(reinterpret_cast<void*>(0x10000), dev));
  const auto type = reinterpret_cast<THPDtype*>(dtype.ptr())->scalar_type;
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(std::move(none), c10::DispatchKeySet(c10::DispatchKey::PrivateUse1),
                                                          c10::scalarTypeToTypeMeta(type));
  t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
  return t;
}

PYBIND11_MODULE(fake_devices, m) {
  m.def("empty", &empty);
  m.def("current", [] { return (int)Fake::getDeviceIndex(); });
  m.def("set_current", [](int i) { Fake::setDeviceIndex(i); });
}
"""

CALLS = r"""
import sys
sys.path.insert(0, sys.argv[1])
sys.path.insert(0, sys.argv[2])
import torch, fake_devices as F
from paper_2608_13966_amd import ops as O
O._load().set_stream_functions(lambda t: seen.append(F.current()) or 0, None)
f32, bf16, i64, u8 = torch.float32, torch.bfloat16, torch.int64, torch.uint8

def e(*shape, dtype=f32):
    return F.empty(list(shape), dtype, at)

for start in (0, 1):
    for at in (0, 1):
        F.set_current(start)
        seen = []
        x, w, n = e(0, 64), e(64), e(0)                 # no rows: nothing is launched
        O.add_rms_norm(x, w, out={"y": x, "rstd": n})
        O.add_rms_norm_backward(x, x, w, n, out={"dx": x}, want_dweight=False)
        i, t, o = e(0, 3, dtype=i64), e(0, 3), {"loss": n, "lse": n, "grad": x}
        O.distill_topk(x, i, t, out=o)
        O.distill_topk_backward(x, i, t, n, out=o)
        O.distill_topk_grad(x, i, t, out=o)
        c, s = e(8 * 64, dtype=u8), e(8)
        O.linear_codes(e(0, 128, dtype=bf16), O.PackedWeight(8, 128, c, s, s), out={"y": e(0, 8, dtype=bf16)})
        print(start, at, seen, F.current())
        assert seen == [at] * 6 and F.current() == start
"""


def test_calls_run_on_their_tensors_device(tmp_path):
    import torch
    from torch.utils import cpp_extension
    src, lib = tmp_path / "fake_devices.cpp", tmp_path / "fake_devices.so"
    src.write_text(DEVICES)
    cmd = [os.environ.get("CXX", "g++"), "-O0", "-std=c++17", "-fPIC", "-shared", "-w",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *[f"-isystem{p}" for p in cpp_extension.include_paths()], f"-isystem{sysconfig.get_paths()['include']}",
           str(src), "-o", str(lib), *[f"-L{p}" for p in cpp_extension.library_paths()], "-lc10", "-ltorch_cpu", "-ltorch",
           "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([sys.executable, "-c", CALLS, ROOT, str(tmp_path)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


@pytest.mark.gpu
def test_a_device_that_is_not_the_current_one():
    import torch
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    from paper_2608_13966_amd import ops as O
    x, w = torch.randn(300, 1000, device="cuda:0"), torch.randn(1000, device="cuda:0")
    want = O.add_rms_norm(x, w, quantize=True)
    with torch.cuda.device(0):
        o = O.add_rms_norm(x.to("cuda:1"), w.to("cuda:1"), quantize=True)
        assert torch.cuda.current_device() == 0 and o["y"].device.index == 1
    assert torch.equal(o["y"].cpu(), want["y"].cpu())
