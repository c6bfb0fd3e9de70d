"""8-bit products of more tiles than one launch takes, checked on the device."""
import pytest
import torch

from paper_2607_16184_amd import ops
from test_gpu_gemm_range import F32, _check, _codes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [3, 30])
def test_weight_rows_past_2_to_27(M):
    N, K = (1 << 27) + 5000, 128
    a, a_s = _codes(M, K), torch.rand(M, 1, device="cuda") + 0.5
    w, w_s = _codes(N, K), torch.rand(-(-N // 128), 1, device="cuda") + 0.5
    y = ops.Linear8(w, w_s).forward(a, a_s)
    for n in range(0, N, 1 << 22):
        _check(y[:, n:n + (1 << 22)], a, a_s, w[n:n + (1 << 22)], w_s[n // 128:(n + (1 << 22)) // 128])
    torch.cuda.empty_cache()


def test_tokens_past_2_to_29():
    M, N, K = (1 << 29) + 300, 3, 128
    a, a_s = _codes(M, K), torch.rand(M, 1, device="cuda") + 0.5
    w, w_s = _codes(N, K), torch.rand(1, 1, device="cuda") + 0.5
    y = ops.Linear8(w, w_s).forward(a, a_s, dtype=F32)
    for m in range(0, M, 1 << 22):
        _check(y[m:m + (1 << 22)], a[m:m + (1 << 22)], a_s[m:m + (1 << 22)], w, w_s)
    torch.cuda.empty_cache()
