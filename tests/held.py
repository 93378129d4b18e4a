"""What matrices held in 8 and 4 bits are, in 64 bits on the CPU: scales, codes and the values that they stand for."""
import torch

GROUP = 64
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
LARGEST = {("f16", 127): 2.0 ** 9, ("f16", 6): 1.328125 * 2.0 ** 13, ("bf16", 127): 2.0 ** 121, ("bf16", 6): 1.328125 * 2.0 ** 125}


def scale64(most, top, type_):
    """The smallest bf16 number, 2^-126 at least, with top * s >= most; NaN where most is not finite."""
    s = (most / top).float().bfloat16()                               # a step beside it at most
    for _ in range(2):
        s = torch.where(top * s.double() < most, (s.view(torch.int16) + 1).view(torch.bfloat16), s)
    below = (s.view(torch.int16) - 1).view(torch.bfloat16)
    s = torch.where((top * below.double() >= most) & (s > 2.0 ** -126), below, s).double()
    s = s.clamp(2.0 ** -126, LARGEST["f16" if type_ == "f16" else "bf16", top])
    return torch.where(torch.isfinite(most), s, torch.full_like(s, float("nan")))


def most64(g):
    """Largest absolute value along the last dimension; infinite where there is an infinity or NaN."""
    return torch.where(torch.isfinite(g), g.abs(), torch.full_like(g, float("inf"))).amax(-1)


def grouped(x, size):
    n, f = x.shape
    return torch.nn.functional.pad(x, (0, -f % size)).view(n, -1, size)


def pack64(x, type_):
    """Codes (n x f) and scales of a checkpoint, in 64 bits; codes of a group that is not finite are 0."""
    g = grouped(x.double(), GROUP)
    s = scale64(most64(g), 127, type_)
    c = torch.nan_to_num((g / s[:, :, None]).round()).clamp(-127, 127)
    c = torch.where(torch.isfinite(s)[:, :, None], c, torch.zeros_like(c))
    return c.view(x.shape[0], -1)[:, :x.shape[1]], s


def unpack64(codes, scales, dtype):
    """The elements that a checkpoint stands for, as 64-bit numbers."""
    s = scales.double().repeat_interleave(GROUP, 1)[:, :codes.shape[1]]
    return (codes.double() * s).to(dtype).double()


def places64(w, s):
    """Places (0 to 7) of |w| / s among LEVELS, each by its distance to all of them; of two that are as near the even one."""
    a = (w.double().abs() / s).unsqueeze(-1)
    far = (a - LEVELS).abs()
    least = far.amin(-1, keepdim=True)
    near = far == least
    even = near & (torch.arange(8) % 2 == 0)
    pick = torch.where(even.any(-1, keepdim=True), even, near)
    return pick.to(torch.int64).argmax(-1)


def pack4_64(w, group, type_):
    """Codes (K x cols, 0 to 15; 0 in a group that is not finite) and scales (groups x cols) of weights in 4 bits."""
    K, cols = w.shape
    g = grouped(w.double().t(), group)
    s = scale64(most64(g), 6, type_)
    place = places64(torch.nan_to_num(g), torch.nan_to_num(s, nan=1.0)[:, :, None])
    code = place + 8 * ((g < 0) & (place > 0))
    code = torch.where(torch.isfinite(s)[:, :, None], code, torch.zeros_like(code))
    return code.view(cols, -1)[:, :K].t(), s.t()


def words4(code):
    """Codes as they lie in memory: eight of a column in a word, the first in its lowest bits."""
    K, cols = code.shape
    c = torch.nn.functional.pad(code, (0, 0, 0, -K % 8)).view(-1, 8, cols)
    w = (c << torch.arange(0, 32, 4)[None, :, None]).sum(1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).int()


def codes4(words, K):
    return ((words.long()[:, None, :] >> torch.arange(0, 32, 4)[None, :, None]) & 15).reshape(-1, words.shape[1])[:K]


def unpack4_64(code, scales, group):
    """The weights that the codes stand for, in 64 bits."""
    v = LEVELS[code & 7]
    return torch.where(code >= 8, -v, v) * scales.double().repeat_interleave(group, 0)[:code.shape[0]]
