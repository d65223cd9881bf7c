"""Products with 4-bit weights: the way out of a wait that runs out in the kernel for few rows."""
import pytest
import torch

from test_gpu_w4 import _bound, _check, _inputs, _weights64, sp  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [1, 5, 16])
def test_a_missing_signal_is_reported(sp, M):  # noqa: F811
    """A CTA's stages are never free again (16384 columns are eight stages of four each, however they are split):
    its loads' wait gives up, the call is reported, nothing is written, and the next call works."""
    ctx = sp.Context(0)
    K, N = 16384, 256
    x, codes, scales, _ = _inputs(M, K, N, 128, False)
    w = sp.W4(ctx, codes.cuda(), scales.cuda())
    y = torch.full((M, N), 7.0, device="cuda")
    ctx.sync()
    ctx.set_wait_limit(20_000_000)
    ctx.set_fault(1)
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y)
    with pytest.raises(sp.SparoaError) as e:
        ctx.sync()
    assert e.value.status == sp.ERR_TIMEOUT
    assert (y == 7).all()  # (nothing is written without sums)
    ctx.set_fault(0)
    ctx.set_wait_limit(0)
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y)
    ctx.sync()
    w64 = _weights64(codes, scales, None, 128)
    _check(y, x.double() @ w64.t(), _bound(x, w64, 128), False, "after a missing signal")
    ctx.close()
