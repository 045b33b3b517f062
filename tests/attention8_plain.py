"""Keys and values of 8 bits from their definition, in 64 bits on the CPU: e4m3 codes with one power of two for each block and key head.

Bounds.  A code stands for y / scale rounded once to the nearest of e4m3's numbers, so what it stands for is off by at most half a step
at y: 2^-4 of |y|'s power of two, and 2^-10 scales where that is less than 2^-6 scales.  Where y itself is computed in float32 with an error of
at most d, the result is off by half a step at |y| + d, and d.  A value that is copied has d = 0: its code is the same bits as
torch's own rounding of y / scale, which is exact in float32.

Attention over codes: the operands are exact in bfloat16 from 2^-133 on and in binary16 from 2^-24 on, so the bounds are those of
attention_plain over the values that the codes stand for.
"""
import math

import torch

CODE, SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu
MOST = {torch.bfloat16: 15 * 2.0 ** 124, torch.float16: 15 * 2.0 ** 12}


def values(codes):
    """Codes as float64."""
    return codes.cpu().float().double()


def scales(scale):
    """Scales as float64: 255 is not a number."""
    byte = scale.cpu().view(torch.uint8).double()
    return torch.where(byte == 255, torch.full_like(byte, math.nan), torch.exp2(byte - 127))


def stands_for(codes, scale):
    """Values [pages][page][kv][dim] of a paged cache."""
    block = codes.shape[1] // scale.shape[1]
    return values(codes) * scales(scale).repeat_interleave(block, 1)[..., None]


def rows_stand_for(codes, scale, block):
    """Values [rows][kv][dim] of rows in blocks."""
    return values(codes) * scales(scale).repeat_interleave(block, 0)[:len(codes), :, None]


def quantised(x, block):
    """Codes and scales of rows x [n][kv][dim] (float32, n a multiple of block), as an empty cache would get them."""
    n, kv, dim = x.shape
    y = x.view(n // block, block, kv, dim)
    byte = ((y.abs().amax((1, 3)).view(torch.int32) >> 23) - 7).clamp(min=1)
    power = ((254 - byte) << 23).view(torch.float32)
    return (y * power[:, None, :, None]).to(CODE).view(n, kv, dim), byte.to(torch.uint8).view(SCALE)


def half_step(size, scale):
    """Half the distance between e4m3's numbers times the scale, at numbers of this size."""
    power = torch.floor(torch.log2((size / scale).clamp(min=2.0 ** -6)))
    return torch.exp2(power - 4) * scale


def runs(pos, slot, n_pos, n_slots, block):
    """[(block, first row, rows)] of a step."""
    at = [s // block if 0 <= p < n_pos and 0 <= s < n_slots else -1 for p, s in zip(pos, slot)]
    out, t = [], 0
    while t < len(at):
        e = t + 1
        while e < len(at) and at[e] == at[t]:
            e += 1
        if at[t] >= 0:
            out.append((at[t], t, e - t))
        t = e
    return out


def check_store(y, d, slot, found, before, after, block, dtype, exact, what=""):
    """Rows y [t][kv][dim] (float64, each within d of what the kernel has) of the runs `found` in the cache `before` = (codes, scales),
    [slots][kv][dim] and [blocks][kv], against `after`.  exact: d is 0, codes are equal bit by bit."""
    codes, byte = (x.clone() for x in before)
    most = MOST[dtype]
    for b, t, n in found:
        first = slot[t] % block
        for c in range(y.shape[1]):
            x = y[t:t + n, c]
            size = torch.where(x.abs() < math.inf, x.abs(), torch.zeros_like(x)).clamp(max=most)
            err = torch.where(x.abs() < math.inf, d[t:t + n, c], torch.zeros_like(x))  # what is not a number has no part in E
            old = int(before[1][b, c]) if first else 0
            low, high = (max(math.floor(math.log2(float(s.max()))) + 120 if float(s.max()) > 0 else 1, 1, old) for s in (size - err, size + err))
            got = int(after[1][b, c])
            assert low <= got <= high, (what, b, c, low, got, high)
            byte[b, c] = got
            scale = 2.0 ** (got - 127)
            if first and got != 255:  # what stands in front, at the new scale; exact in float32
                held = codes[b * block:b * block + first, c]
                held.view(torch.uint8).copy_((held.float() * 2.0 ** max(old - got, -149)).to(CODE).view(torch.uint8))
            at = torch.tensor(slot[t:t + n])
            now = after[0][at, c]
            want = torch.where(x.abs() < math.inf, x.clamp(-most, most), torch.full_like(x, math.nan))
            off = (values(now) * scale - want).abs()
            bound = half_step(size + err, scale) + err
            assert bool((off[want == want] <= bound[want == want]).all()), (what, b, c, float((off - bound)[want == want].max()))
            assert torch.isnan(values(now)[want != want]).all(), (what, b, c)
            if exact:
                mine = (want.float() * 2.0 ** (127 - got)).to(CODE)
                same = (mine.view(torch.uint8) == now.view(torch.uint8)) | (mine.float().isnan() & now.float().isnan())
                assert bool(same.all()), (what, b, c)
            codes[at, c] = now
    assert torch.equal(codes.view(torch.uint8), after[0].view(torch.uint8)), what  # all else as it was
    assert torch.equal(byte, after[1]), what
