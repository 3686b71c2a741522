"""Values held in 8-bit floating point with a power of two for each 128, by the definition: on the CPU, in
64 bits."""

import torch


def e4m3(v):
    """The nearest value of e4m3, ties to even, of |v| <= 448 (float64): steps of 2^-3 of the octave,
    2^-9 below 2^-6."""
    _, octave = torch.frexp(v.abs().clamp_min(2.0 ** -6))
    step = torch.ldexp(torch.ones_like(v), octave - 1 - 3)
    return torch.round(v / step) * step


def hold(x, square=False):
    """(q as float64 values, bytes [rows][blocks]) of x [rows][width]."""
    x = x.double()
    rows, width = x.shape
    blocks, tall = -(-width // 128), -(-rows // 128)
    room = torch.zeros(tall * 128, blocks * 128, dtype=torch.float64)
    room[:rows, :width] = x
    tiles = room.view(tall, 128, blocks, 128)
    bad = ~torch.isfinite(tiles)
    size = torch.where(bad, torch.inf, tiles.abs())
    top = size.amax((1, 3) if square else 3, keepdim=True).expand(tall, 128, blocks, 1)
    nan = torch.isinf(top)
    e = torch.full(top.shape, -127.0, dtype=torch.float64)
    for _ in range(2):  # a start one below the answer at most, then up by one where that is too small
        start = torch.frexp((top / 448).clamp(2.0 ** -127, 2.0 ** 127))[1].double() - 2
        e = torch.maximum(e, start)
    for _ in range(2):
        e = torch.where((top > 448 * torch.ldexp(torch.ones_like(e), e)) & ~nan, e + 1, e)
    q = torch.where(nan, 0.0, e4m3(torch.where(nan, 0.0, tiles) * torch.ldexp(torch.ones_like(e), -e)))
    byte = torch.where(nan, 255.0, e + 127).to(torch.int64)
    return (q.reshape(room.shape)[:rows, :width],
            byte.reshape(tall * 128, blocks)[:rows])


def values(q, byte):
    """q 2^(byte - 127), NaN where the byte is 255."""
    unit = torch.ldexp(torch.ones(byte.shape, dtype=torch.float64), byte - 127)
    unit = torch.where(byte == 255, torch.nan, unit)
    return q.double() * unit.repeat_interleave(128, 1)[:, :q.shape[1]]


def in_order(byte):
    """Bytes [rows][blocks] in the kernels' order, [blocks][rows up to 128], by its formula."""
    rows, blocks = byte.shape
    out = torch.zeros(blocks, -(-rows // 128) * 128, dtype=torch.uint8)
    i = torch.arange(rows)
    out[:, i // 128 * 128 + i % 16 * 8 + i % 128 // 16] = byte.t().to(torch.uint8)
    return out


def scaled(kr, x, square=False):
    """x held by this file, as the library's Scaled on the device: contiguous rows."""
    q, byte = hold(x, square)
    return kr.Scaled(q.to(torch.float8_e4m3fn).cuda(), in_order(byte).cuda())
