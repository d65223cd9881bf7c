"""Products with 4-bit weights on the GPU against 64 bits.

Tolerances.  Codes less zeros and their products with bf16 x are exact in fp32.  The sum over a group has
at most 128 additions, each off by at most 2^-23 of the terms' sizes (tensor cores may cut instead of
rounding), the sum over the K / 32 groups at most and up to 8 parts by 2^-24 each: (2^-16 + (K / 32 + 8)
2^-24) of sum |x w|.  Bias, residual and the affine form add four roundings, 2^-22 of their terms; a bf16
result is rounded once, 2^-8 of its size."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2511_19457_gb300 import sparoa
    return sparoa


@pytest.fixture(scope="module")
def ctx(sp):
    c = sp.Context(0)
    yield c
    c.sync()
    c.close()


def _inputs(M, K, N, group, zeros, seed=0):
    g = torch.Generator().manual_seed(seed * 7919 + M * 31 + K + N)
    x = torch.randn(M, K, generator=g).to(torch.bfloat16)
    codes = torch.randint(0, 256, (N, K // 2), generator=g).to(torch.uint8)
    scales = (torch.randn(N, K // group, generator=g) * 0.1).to(torch.bfloat16)
    zero = torch.randint(0, 16, (N, K // group), generator=g).to(torch.uint8) if zeros else None
    return x, codes, scales, zero


def _weights64(codes, scales, zero, group):
    N, K = codes.shape[0], codes.shape[1] * 2
    c = torch.stack([codes & 15, codes >> 4], -1).view(N, K).double()
    z = zero.double().repeat_interleave(group, 1) if zero is not None else 8.0
    return (c - z) * scales.double().repeat_interleave(group, 1)


def _bound(x, w, group):
    K = x.shape[1]
    return (2.0 ** -16 + (K / 32 + 8) * 2.0 ** -24) * (x.double().abs() @ w.abs().t())


def _check(got, want, tol, bf16, what):
    got = got.double().cpu()
    tol = tol + (2.0 ** -8 * want.abs() if bf16 else 2.0 ** -22 * want.abs())
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {((got - want).abs() - tol).max():.3e}"


def _run(sp, ctx, M, K, N, group, zeros, out, seed=0):
    x, codes, scales, zero = _inputs(M, K, N, group, zeros, seed)
    w = sp.W4(ctx, codes.cuda(), scales.cuda(), None if zero is None else zero.cuda())
    y = torch.full((M, N), float("nan"), dtype=out, device="cuda")
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y)
    w64 = _weights64(codes, scales, zero, group)
    _check(y, x.double() @ w64.t(), _bound(x, w64, group), out == torch.bfloat16, f"{M} {K} {N} {group}")


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 33, 61, 64, 65, 130])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_rows(sp, ctx, M, group, zeros):
    _run(sp, ctx, M, 5 * 128 + group, 264, group, zeros, torch.float32)


@pytest.mark.parametrize("M", [66, 127, 128, 129, 192, 300])
@pytest.mark.parametrize("K,N,group,zeros", [(96, 24, 32, True), (1024, 2048, 64, False), (4096, 1000, 128, True), (640, 5000, 32, False)])
def test_many_rows(sp, ctx, M, K, N, group, zeros):
    _run(sp, ctx, M, K, N, group, zeros, torch.float32)


@pytest.mark.parametrize("K,N,group", [(32, 8, 32), (64, 8, 64), (128, 16, 128), (160, 24, 32), (352, 128, 32), (384, 136, 128), (448, 1000, 64),
                                       (1024, 2048, 128), (2048, 520, 128), (4000, 72, 32), (16384, 64, 128), (256, 16384, 64), (8192, 1032, 32)])
@pytest.mark.parametrize("M", [1, 5, 16, 40])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_sizes(sp, ctx, K, N, group, M, out):
    """Columns that end inside a tile, rows that end inside one, one tile to many, every way of splitting."""
    _run(sp, ctx, M, K, N, group, K % 3 == 1, out)


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("bias,bn,residual", [(True, False, False), (False, True, True), (True, True, True)])
@pytest.mark.parametrize("M,out", [(3, torch.bfloat16), (37, torch.float32)])
def test_epilogue(sp, ctx, act, bias, bn, residual, M, out):
    K, N, group = 512, 328, 64
    x, codes, scales, zero = _inputs(M, K, N, group, True)
    g = torch.Generator().manual_seed(5)
    b = torch.randn(N, generator=g) if bias else None
    stats = torch.stack([torch.rand(N, generator=g) + 0.5, torch.randn(N, generator=g), torch.randn(N, generator=g), torch.rand(N, generator=g) + 0.5]) if bn else None
    r = torch.randn(M, N, generator=g).to(torch.bfloat16) if residual else None
    w = sp.W4(ctx, codes.cuda(), scales.cuda(), zero.cuda())
    y = torch.empty(M, N, dtype=out, device="cuda")
    occ = sp.OccupancyBuffer(M, N) if out == torch.bfloat16 else None
    dev = [None if t is None else t.cuda() for t in (b, stats, r)]
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y, bias=dev[0], bn=dev[1], act=act, residual=dev[2], y_occ=occ)
    w64 = _weights64(codes, scales, zero, group)
    want, tol = x.double() @ w64.t(), _bound(x, w64, group)
    size = want.abs()
    if bias:
        want, size = want + b.double(), size + b.double().abs()
    if bn:
        gamma, beta, mean, var = stats.double()
        k = gamma / (var + 1e-5).sqrt()
        want, size, tol = (want - mean) * k + beta, (size + mean.abs()) * k.abs() + beta.abs(), tol * k.abs()
    if residual:
        want, size = want + r.double(), size + r.double().abs()
    if act:
        want = want.clamp_min(0)
    if act == 2:
        want = want.clamp_max(6)
    _check(y, want, tol + 2.0 ** -20 * size, out == torch.bfloat16, "epilogue")
    if occ:
        assert occ.to_host()["nnz"] == int((y != 0).sum())


def test_in_place_of_the_residual(sp, ctx):
    M, K, N = 5, 256, 64
    x, codes, scales, _ = _inputs(M, K, N, 128, False)
    w = sp.W4(ctx, codes.cuda(), scales.cuda())
    r = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    y = r.cuda()
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y, residual=y)
    w64 = _weights64(codes, scales, None, 128)
    _check(y, x.double() @ w64.t() + r.double(), _bound(x, w64, 128), True, "in place")


def test_extreme_codes_and_values(sp, ctx):
    """Codes 0 and 15 against zeros 0 and 15, scales of zero and far from 1, a row of x that is not finite only
    in its own results."""
    M, K, N, group = 9, 256, 64, 32
    x, codes, scales, zero = _inputs(M, K, N, group, True)
    codes[0], codes[1], codes[2] = 0, 255, 0xF0
    zero[0], zero[1] = 15, 0
    scales[3], scales[4], scales[5] = 0, 2.0 ** 60, 2.0 ** -100
    x[4, 7] = float("nan")
    x[6, 9] = float("inf")
    w = sp.W4(ctx, codes.cuda(), scales.cuda(), zero.cuda())
    y = torch.empty(M, N, device="cuda")
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y)
    fine = [i for i in range(M) if i not in (4, 6)]
    w64 = _weights64(codes, scales, zero, group)
    _check(y[fine], x[fine].double() @ w64.t(), _bound(x[fine], w64, group) + 1e-38, False, "extremes")
    assert y[4].isnan().all() and (~y[6].isfinite()).any()


def test_quantise(sp, ctx):
    """The nearest codes: off by half a step where the range holds the value, and by the rounding of the scale to
    bf16 (2^-8 of 8 steps at the range's ends; a whole step is allowed for both)."""
    g = torch.Generator().manual_seed(2)
    weight = torch.randn(40, 256, generator=g)
    weight[3] = 0
    for zeros in (False, True):
        codes, scales, zero = sp.w4_quantise(weight, 64, zeros)
        err = (_weights64(codes, scales, zero, 64) - weight.double()).abs()
        assert (err <= scales.double().repeat_interleave(64, 1) + 1e-12).all()
    x = torch.randn(3, 256, generator=g).to(torch.bfloat16)
    w = sp.W4.quantise(ctx, weight.cuda(), 64)
    y = torch.empty(3, 40, device="cuda")
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y)
    codes, scales, zero = sp.w4_quantise(weight, 64)
    w64 = _weights64(codes, scales, zero, 64)
    _check(y, x.double() @ w64.t(), _bound(x, w64, 64), False, "quantised")


def test_streams_and_graphs(sp, ctx):
    """Replayed on other values and on another stream; results are the same bits, run after run."""
    M, K, N = 6, 1024, 512
    x, codes, scales, _ = _inputs(M, K, N, 128, False)
    w = sp.W4(ctx, codes.cuda(), scales.cuda())
    xd, y = x.cuda(), torch.empty(M, N, device="cuda")
    sp.sparoa_gemm_w4(ctx, xd, w, y)
    first = y.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.sparoa_gemm_w4(ctx, xd, w, y)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, first)
    x2 = torch.randn(M, K, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    xd.copy_(x2)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        graph.replay()
    torch.cuda.synchronize()
    w64 = _weights64(codes, scales, None, 128)
    _check(y, x2.double() @ w64.t(), _bound(x2, w64, 128), False, "replayed")


def test_waits_end(sp):
    """A wait whose limit is a cycle gives up and is reported, or was over at once; the context works on."""
    ctx = sp.Context(0)
    x, codes, scales, _ = _inputs(4, 2048, 256, 128, False)
    w = sp.W4(ctx, codes.cuda(), scales.cuda())
    y = torch.empty(4, 256, device="cuda")
    ctx.sync()
    ctx.set_wait_limit(1)
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y)
    try:
        ctx.sync()
    except sp.SparoaError as e:
        assert e.status == sp.ERR_TIMEOUT
    ctx.set_wait_limit(0)
    sp.sparoa_gemm_w4(ctx, x.cuda(), w, y)
    ctx.sync()
    w64 = _weights64(codes, scales, None, 128)
    _check(y, x.double() @ w64.t(), _bound(x, w64, 128), False, "after a timeout")
    ctx.close()


@pytest.mark.parametrize("M", [40, 128])
def test_a_missing_signal_is_reported(sp, M):
    """The tensor cores' signal withheld: the wait for it gives up, the call is reported, and the next one works."""
    ctx = sp.Context(0)
    x, codes, scales, _ = _inputs(M, 1024, 256, 128, False)
    w = sp.W4(ctx, codes.cuda(), scales.cuda())
    y = torch.full((M, 256), 7.0, device="cuda")
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


@pytest.mark.parametrize("M", [5, 50])
def test_two_streams_at_once(sp, ctx, M):
    """Calls of one context on two streams whose work overlaps: nothing is shared between them."""
    K, N = 2048, 4096
    x, codes, scales, _ = _inputs(M, K, N, 64, False)
    w = sp.W4(ctx, codes.cuda(), scales.cuda())
    x2 = torch.randn(M, K, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    jobs = [(v, v.cuda(), torch.empty(M, N, device="cuda"), torch.cuda.Stream()) for v in (x, x2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for _, v, y, st in jobs:
            with torch.cuda.stream(st):
                sp.sparoa_gemm_w4(ctx, v, w, y)
    torch.cuda.synchronize()
    w64 = _weights64(codes, scales, None, 64)
    for v, _, y, _ in jobs:
        _check(y, v.double() @ w64.t(), _bound(v, w64, 64), False, "streams")


def test_rows_behind_are_left(sp, ctx):
    """Results of fewer rows than a tile of tokens write nothing else."""
    for M in (3, 20):
        x, codes, scales, _ = _inputs(M, 256, 72, 32, False)
        w = sp.W4(ctx, codes.cuda(), scales.cuda())
        whole = torch.full((M + 4, 72), 9.0, device="cuda")
        sp.sparoa_gemm_w4(ctx, x.cuda(), w, whole[:M])
        assert (whole[M:] == 9).all() and (whole[:M] != 9).all()


def test_refusals_of_pack(sp, ctx):
    _, codes, scales, zero = (None if t is None else t.cuda() for t in _inputs(4, 256, 64, 64, True))
    packed = torch.empty(sp.W4(ctx, codes, scales, zero).packed.numel(), dtype=torch.uint8, device="cuda")
    bad = [(codes, scales, zero, packed[16:]), (codes, scales, zero, packed.cpu()), (codes, scales, None, packed), (codes, scales[:, :0], None, packed),
           (codes, scales, zero, packed.view(torch.int32)), (codes.int(), scales, zero, packed), (codes, scales, zero[:32], packed)]
    for i, args in enumerate(bad):
        with pytest.raises(sp.SparoaError):
            sp.sparoa_w4_pack(ctx, *args)
            raise AssertionError(f"call {i} was taken")
    sp.sparoa_w4_pack(ctx, codes, scales, zero, packed)
    assert torch.equal(packed, sp.W4(ctx, codes, scales, zero).packed)


def test_refusals(sp, ctx):
    x, codes, scales, zero = (None if t is None else t.cuda() for t in _inputs(4, 256, 64, 64, True))
    w = sp.W4(ctx, codes, scales, zero)
    y = torch.empty(4, 64, device="cuda")
    bad = [lambda: sp.W4(ctx, codes.int(), scales), lambda: sp.W4(ctx, codes, scales.float()), lambda: sp.W4(ctx, codes, scales[:, :1]),
           lambda: sp.W4(ctx, codes[:60], scales[:60]), lambda: sp.W4(ctx, codes, scales, zero[:, :2].contiguous()),
           lambda: sp.W4(ctx, codes, scales.cpu()), lambda: sp.W4(ctx, codes[:, :120], scales),
           lambda: sp.sparoa_gemm_w4(ctx, x[:, :128], w, y), lambda: sp.sparoa_gemm_w4(ctx, x.float(), w, y),
           lambda: sp.sparoa_gemm_w4(ctx, x, w, y[:3]), lambda: sp.sparoa_gemm_w4(ctx, x, w, y.half()),
           lambda: sp.sparoa_gemm_w4(ctx, x, w, y, bias=y[0, :32]), lambda: sp.sparoa_gemm_w4(ctx, x, w, y, residual=y),
           lambda: sp.sparoa_gemm_w4(ctx, x, w, y, act=7), lambda: sp.sparoa_gemm_w4(ctx, x, w, y, y_occ=sp.OccupancyBuffer(4, 64))]
    for i, f in enumerate(bad):
        with pytest.raises(sp.SparoaError):
            f()
            raise AssertionError(f"call {i} was taken")
    sp.sparoa_gemm_w4(ctx, x[:0], w, y[:0])  # no rows: nothing to do
    ctx.sync()
