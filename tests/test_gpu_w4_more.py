"""Products with 4-bit weights: the way out of a wait that runs out in the kernel for few rows, and GELU behind both."""
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


@pytest.mark.parametrize("M,out", [(3, torch.bfloat16), (37, torch.float32), (100, torch.bfloat16)])
def test_gelu(sp, M, out):  # noqa: F811
    """The tanh form, whose slope is 1.13 at most; the hardware's tanh is off by 2^-11 of itself, which is 2^-12 of |x|
    here; as much again is allowed for the form's other roundings."""
    ctx = sp.Context(0)
    K, N, group = 512, 328, 64
    x, codes, scales, zero = _inputs(M, K, N, group, True)
    b = torch.randn(N, generator=torch.Generator().manual_seed(5))
    w = sp.W4(ctx, codes.cuda(), scales.cuda(), zero.cuda())
    y = torch.empty(M, N, dtype=out, device="cuda")
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y, bias=b.cuda(), act=sp.ACT_GELU)
    ctx.sync()
    w64 = _weights64(codes, scales, zero, group)
    z = x.double() @ w64.t() + b.double()
    want = torch.nn.functional.gelu(z, approximate="tanh")
    _check(y, want, 1.13 * (_bound(x, w64, group) + 2.0 ** -22 * z.abs()) + 2.0 ** -11 * z.abs(), out == torch.bfloat16, "gelu")
    ctx.close()


@pytest.mark.parametrize("M", [4, 40, 128])
def test_waits_of_a_cycle(sp, M):  # noqa: F811
    """Waits that give up at once, wherever a call is: reported or not needed, call after call, and then results are
    right."""
    ctx = sp.Context(0)
    x, codes, scales, _ = _inputs(M, 2048, 1024, 128, False)
    w = sp.W4(ctx, codes.cuda(), scales.cuda())
    y = torch.empty(M, 1024, device="cuda")
    xd = x.cuda()
    ctx.sync()
    ctx.set_wait_limit(1)
    for _ in range(10):
        sp.sparoa_gemm_w4(ctx, xd, w, y)
        try:
            ctx.sync()
        except sp.SparoaError as e:
            assert e.status == sp.ERR_TIMEOUT
    ctx.set_wait_limit(0)
    sp.sparoa_gemm_w4(ctx, xd, w, y)
    ctx.sync()
    w64 = _weights64(codes, scales, None, 128)
    _check(y, x.double() @ w64.t(), _bound(x, w64, 128), False, "after waits that gave up")
    ctx.close()
