"""The eigenvector call gives the same bits whatever its workspace and the compute units' LDS held before, and whatever runs beside it."""
import ctypes

import pytest
import torch

from paper_2510_24273_amd import binding
from tests import gpu_util as gu
from tests.test_gpu_calibration import _spectrum_on_device

pytestmark = pytest.mark.gpu


def _call(C, r, fill):
    D = C.shape[0]
    rows = C.clone()
    nbytes = int(binding._lib.sals_calib_eigenvectors_workspace_bytes(D))
    ws = torch.full((nbytes,), fill, dtype=torch.uint8, device=gu.DEV)
    lam = torch.full((8 * D,), fill, dtype=torch.uint8, device=gu.DEV).view(torch.float64)
    U = torch.full((4 * D * r,), fill, dtype=torch.uint8, device=gu.DEV).view(torch.float32).view(D, r)
    sweeps = ctypes.c_int32(0)
    st = binding._lib.sals_calib_eigenvectors(rows.data_ptr(), D, r, binding.SALS_F32, lam.data_ptr(), U.data_ptr(), ws.data_ptr(), nbytes, 80,
                                              ctypes.byref(sweeps), torch.cuda.current_stream().cuda_stream)
    assert binding.status_string(st) == "SALS_OK"
    torch.cuda.synchronize()
    return rows, lam, U, sweeps.value


@pytest.mark.parametrize("D,r,decay,mixed", [(256, 160, 0.25, True), (512, 512, 1.0, False), (1024, 640, 0.25, True), (1024, 512, 1.0, False),
                                             (1280, 800, 0.25, True), (2048, 1280, 0.25, True), (2048, 256, 1.0, False), (2816, 500, 0.25, True)])
def test_the_call_repeats_whatever_memory_held_and_beside_other_work(D, r, decay, mixed):
    print(f"[case] eigenvectors after other contents and beside other work, D={D} r={r} decay={decay}", flush=True)
    C = _spectrum_on_device(D, decay, mixed)
    first = _call(C, r, 0)
    nan_keys = torch.full((8192, 2048), float("nan"), dtype=torch.bfloat16, device=gu.DEV)
    side, a = torch.cuda.Stream(), torch.ones(1 << 26, device=gu.DEV)
    b = torch.empty_like(a)
    for fill, dirty, beside in ((0xFF, False, False), (0xA5, True, False), (0, True, True), (0x3C, False, True), (0xFF, True, True)):
        if dirty:   # (128 KB of LDS of every compute unit are left as NaN)
            binding.calib_accumulate(nan_keys, torch.zeros(2048, 2048, dtype=torch.float64, device=gu.DEV))
            torch.cuda.synchronize()
        if beside:  # (two launches at a time: the device's memory is busy while the call runs)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                for _ in range(40):
                    b.copy_(a)
        again = _call(C, r, fill)
        assert again[3] == first[3], (fill, dirty, beside)
        for x, y in zip(again[:3], first[:3]):
            assert torch.equal(x, y), (fill, dirty, beside)
