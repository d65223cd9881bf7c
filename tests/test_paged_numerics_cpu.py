"""Models of the attention kernels' rounding on the CPU: what the bounds of the GPU tests tell apart."""
import torch


def test_one_part_of_a_weight_would_show():
    """The bound on results of few rows (2^-14 of sum p |v|) tells weights of two bf16 parts from one."""
    g = torch.Generator().manual_seed(1)
    x = (1 + 0.5 * torch.rand(200, generator=g)).to(torch.bfloat16).double() / 32  # the scores' difference
    w = torch.exp(-x)
    want = (1 - w) / (1 + w)
    tol = 2.0 ** -8 * want + 2.0 ** -14
    hi = w.float().to(torch.bfloat16).double()
    lo = (w - hi).float().to(torch.bfloat16).double()
    assert (((1 - hi - lo) / (1 + w) - want).abs() <= tol / 4).all()
    assert (((1 - hi) / (1 + w) - want).abs() > tol).double().mean() > 0.5
