"""What the tests of the losses share: inputs, and the definitions in 64 bits with bounds on what 32 bits may be off."""
import torch

from paper_2602_05145_amd import binding as B

DEV = "cuda:0"
TDT = {"fp32": torch.float32, "bf16": torch.bfloat16}
CODE = {"fp32": B.TIDE_DTYPE_FP32, "bf16": B.TIDE_DTYPE_BF16}
HALF = 2.0 ** -24                       # half a step of fp32, relative
STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}   # rounding of a stored result, relative


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def logits(rows, vocab, ldz, dtype, seed, scale=3.0):
    """[rows, ldz] of which the columns from vocab on hold NaN: nothing may look at them."""
    z = torch.full((rows, ldz), float("nan"), device=DEV, dtype=TDT[dtype])
    z[:, :vocab] = scale * torch.randn((rows, vocab), device=DEV, generator=gen(seed))
    return z


def padded(vocab, extra=0):
    return (vocab + 7) // 8 * 8 + extra


def sum_rel(n, reach):
    """Relative error of a sum of n exponentials exp(x), each as a power of two from one fused step, in fp32: at most n / 256 + 64 roundings
    follow each other (256 threads or more share a row), the largest term's exponent comes from numbers up to `reach`, which the rounded
    1 / ln 2 and the rounded shift move by 2 |reach| half steps, and the instruction itself is good to a step."""
    return (n / 256 + 64 + 4 * reach) * HALF


def lse64(z, tau):
    """(log-sum-exp of z / tau in 64 bits, what fp32 may be off): the sum's relative error, and the roundings of max / tau, log and their sum."""
    x = z.double() / tau
    lse = torch.logsumexp(x, 1)
    reach = x[x.isfinite()].abs().max() if x.isfinite().any() else torch.tensor(0.0)
    return lse, sum_rel(z.shape[1], float(reach)) + 4 * HALF * (float(reach) + 16)


def assert_within(got, want, tol, what):
    """|got - want| <= tol everywhere, and the same infinities and NaN."""
    got, want = got.double(), want.double()
    tol = torch.as_tensor(tol, dtype=torch.float64, device=want.device).expand_as(want)
    fine = want.isfinite()
    assert torch.equal(got.isnan(), want.isnan()), what
    assert torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()]), what
    over = (got[fine] - want[fine]).abs() - tol[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, "over by", float(over.max()), "of", float(tol[fine].max()))
