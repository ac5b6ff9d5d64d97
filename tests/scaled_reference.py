"""Plain 64-bit definitions of the 8-bit block-scaled operators and of rows sorted by expert, for the tests: torch on any device."""
import torch

BLOCK = 128
TOP = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
GRID = {torch.float8_e4m3fn: (3, -6), torch.float8_e5m2: (2, -14)}      # fraction bits, least exponent


def power(e):
    """2^e in 64 bits for whole e."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def scale_values(scale):
    """Scales in 64 bits: float32 as they are, E8M0 bytes as powers of two (255: NaN)."""
    if scale.dtype == torch.float32:
        return scale.double()
    b = scale.view(torch.uint8).to(torch.int64)
    return torch.where(b == 255, torch.nan, power(b - 127))


def dequantize(data, scale, cols, block_rows):
    """What an 8-bit matrix (rows x at least cols) with its scales stands for, in 64 bits."""
    x = data[..., :cols].to(torch.float32).double()
    c = torch.arange(cols, device=x.device) // BLOCK
    r = torch.arange(x.shape[-2], device=x.device) // block_rows
    return x * scale_values(scale)[..., r, :][..., c]


def exponents(x, dtype, block_rows):
    """Exponent of each block's scale by exhaustive comparison: the least e in [-126, 127] with max |x| <= TOP 2^e; 0 for zeros;
    128 marks a block with an infinity or a NaN."""
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // BLOCK)
    full = torch.zeros((nr * block_rows, nc * BLOCK), dtype=torch.float64, device=x.device)
    full[:rows, :cols] = x.double().abs()
    top = full.view(nr, block_rows, nc, BLOCK).amax(dim=(1, 3))
    ladder = torch.arange(-126, 128, device=x.device)
    e = 127 - (top.unsqueeze(-1) <= TOP[dtype] * power(ladder)).sum(-1) + 1
    e = torch.where(top == 0, 0, e)
    return torch.where(torch.isfinite(top), e, 128)


def round_to(x, dtype):
    """Nearest value of the 8-bit type, ties to even, in 64 bits (|x| within the type's range)."""
    frac, low = GRID[dtype]
    step = power((torch.frexp(x).exponent - 1).clamp(min=low) - frac)
    return torch.round(x / step) * step


def quantize(x, dtype, block_rows):
    """(values on the 8-bit grid, exponents): NaN throughout a block without a scale."""
    e = exponents(x, dtype, block_rows)
    r = torch.arange(x.shape[0], device=x.device) // block_rows
    c = torch.arange(x.shape[1], device=x.device) // BLOCK
    each = e[r][:, c]
    v = round_to(torch.where(each == 128, 0.0, x.double()) * power(-each.clamp(max=127)), dtype)
    return torch.where(each == 128, torch.nan, v), e


def sort_choices(ids, experts):
    """(offsets, order, place) by a loop over the choices."""
    flat = ids.reshape(-1).tolist()
    by = [[] for _ in range(experts)]
    for i, e in enumerate(flat):
        if 0 <= e < experts:
            by[e].append(i)
    offsets, order = [0], []
    for b in by:
        order += b
        offsets.append(len(order))
    place = [-1] * len(flat)
    for s, i in enumerate(order):
        place[i] = s
    order += [-1] * (len(flat) - len(order))
    return offsets, order, place
