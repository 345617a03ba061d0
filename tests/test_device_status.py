"""npd_device_status: a bounded wait that ran out is seen without the status word of the call it happened in."""

import pytest
import torch

from paper_2605_05940_b200 import binding as B
from paper_2605_05940_b200 import build as npd_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    npd_build.build()


def test_refusals_on_the_host():
    assert B.lib().npd_device_status(None, None) == B.NPD_EINVAL


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the behaviour on a box without a GPU")
def test_without_a_gpu_it_says_so():
    import ctypes as C
    out = C.c_int32(7)
    assert B.lib().npd_device_status(None, C.byref(out)) == B.NPD_ECUDA and out.value == 7


@pytest.mark.gpu
def test_a_wait_that_ran_out_stays_until_it_is_read():
    # the self-test's wait ends after 2e5 cycles and reports as the tensor kernels do (report_timeout)
    B.npd_device_status()
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda n, m: torch.randn((n, m), device="cuda", generator=g).to(torch.bfloat16)
    x, w, dy = r(300, 128), r(200, 128), r(300, 200)

    def work():
        B.npd_linear_fwd(x, w)
        B.npd_linear_bwd(dy, x, w)
        B.npd_gemm_bf16(x, w, torch.empty((300, 200), device="cuda"))
        B.npd_cross_entropy(x, w, torch.randint(0, 200, (300,), device="cuda", dtype=torch.int32))

    work()
    assert B.npd_device_status() == B.NPD_OK
    B.npd_selftest_wait_timeout(200_000)
    work()                                                    # nothing of this clears the word
    assert B.npd_device_status("cuda") == B.NPD_ETIMEOUT
    assert B.npd_device_status("cuda:0") == B.NPD_OK
    side = torch.cuda.Stream()
    B.npd_selftest_wait_timeout(200_000, stream=side)
    assert B.npd_device_status(stream=side) == B.NPD_ETIMEOUT and B.npd_device_status(0) == B.NPD_OK
