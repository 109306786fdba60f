"""4-bit products whose sums are exact in fp32 in any order: the output is the one rounding of a whole
number, equal bit for bit, so that a lost column, a scale of its neighbour or a weight rounded to bf16
is seen at every width, where a bound on sums of thousands of terms would pass it.

x is +-1 or +-2, codes are any, scales are odd whole numbers of 9 bits (fp32, one more bit than bf16
holds) or 8 (bf16), times `unit`.  Within a group all sums stay below 31 * 2 * 128; over the groups they
are multiples of `unit` below 2^24 of them, which `product` checks."""
import torch


def rows(g, M, K, device):
    x = torch.randint(1, 3, (M, K), device=device, generator=g)
    return (x * (2 * torch.randint(0, 2, (M, K), device=device, generator=g) - 1)).to(torch.bfloat16)


def matrix(g, *lead, K, group, scale, device, unit=1):
    codes = torch.randint(0, 256, (*lead, K // 2), dtype=torch.uint8, device=device, generator=g)
    lo = 64 if scale is torch.bfloat16 else 128
    s = 2 * torch.randint(lo, 2 * lo, (*lead, K // group), device=device, generator=g) + 1
    s *= 2 * torch.randint(0, 2, s.shape, device=device, generator=g) - 1
    return codes, (s * unit).to(scale)


def product(x, codes, scale, group, unit=1):
    """x W^T in float64, exact, after showing that fp32 holds every partial sum."""
    q = torch.stack((codes % 16, codes // 16), -1).flatten(-2).double() - 8
    y, size = (torch.zeros(len(x), len(codes), dtype=torch.float64, device=x.device) for _ in range(2))
    for i in range(scale.shape[-1]):
        at = slice(i * group, (i + 1) * group)
        p = (x[:, at].double() @ q[:, at].T.contiguous()) * scale[:, i].double()
        y += p
        size += p.abs()
    assert bool((size < unit * 2.0 ** 24).all())
    return y


GATE_UNIT = 128   # a gate sum is 0 or at least 128 either way, where SiLU in fp32 is max(v, 0): exp(-128)
                  # is no fp32 number but 0 beside 1, and exp(128) is past the largest


def swiglu(gate, up):
    """Both exact in fp32: one rounding of their product, then the output's."""
    return (gate.clamp(min=0).float() * up.float()).to(torch.bfloat16)
