"""64-bit reference of the 4-bit cache: every code by trying all of them."""
import torch

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantise(x):
    """x [..., D] on the CPU: codes [..., D/2] and bytes [..., D/32], uint8."""
    a = x.double().unflatten(-1, (-1, 32))
    top = a.abs().amax(-1)
    # the smallest power of two that the largest magnitude fits under, found by trying them all
    e = torch.arange(-124, 126)
    fits = top.unsqueeze(-1) <= 7.0 * torch.ldexp(torch.ones(()).double(), e)
    fits[..., -1] = True
    e = e[fits.int().argmax(-1)]
    y = torch.ldexp(a, -e.unsqueeze(-1))
    far = (y.abs().unsqueeze(-1) - LEVELS).abs()
    near = far == far.amin(-1, keepdim=True)
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(-1), even.int().argmax(-1), near.int().argmax(-1))
    code = (code + 8 * torch.signbit(a)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def values(codes, scales):
    """The 64-bit values of codes and bytes, wherever they lie."""
    lv = torch.cat([LEVELS, -LEVELS]).to(codes.device)
    v = torch.stack([lv[(codes % 16).long()], lv[(codes // 16).long()]], -1).flatten(-2)
    return v * torch.exp2(scales.double() - 127.0).repeat_interleave(32, -1)
