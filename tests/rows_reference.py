"""Rows of latent attention in 64 bits: the formats, avsg_append's quantisation and avsg_attend, from their definitions."""
import math

import torch

LATENT, ROPE = 512, 64
BYTES = {0: 1152, 1: 656, 2: 400}
E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def random_rows(shape, fmt, gen, device, spread=0.5):
    """Packed rows whose magnitudes differ by row."""
    n = math.prod(shape)
    x = torch.randn(n, LATENT, generator=gen, device=device) * torch.exp(spread * torch.randn(n, 1, generator=gen, device=device))
    r = torch.randn(n, ROPE, generator=gen, device=device).to(torch.bfloat16)
    return pack(x.double(), r, fmt).view(*shape, BYTES[fmt])


def groups_to_nearest(v, mantissa, least, most):
    """To the nearest number of so many mantissa bits, ties to even, steps no finer than at 2^least, largest magnitude `most`."""
    e = torch.frexp(v).exponent - 1
    step = torch.ldexp(torch.ones_like(v), e.clamp(min=least) - mantissa)
    return (torch.round(v / step) * step).clamp(-most, most)


def pack(x, rope, fmt):
    """fp64 latents [n, 512] and bf16 [n, 64] -> uint8 rows, as avsg_append defines them."""
    n = x.shape[0]
    tail = rope.contiguous().view(torch.uint8).view(n, 128)
    if fmt == 0:
        return torch.cat((x.float().to(torch.bfloat16).view(torch.uint8).view(n, 1024), tail), 1)
    if fmt == 1:
        g = x.view(n, 4, 128)
        scale = (g.abs().amax(2) / 448.0).float().clamp(min=2.0 ** -126)
        v = groups_to_nearest(g / scale.double()[..., None], 3, -6, 448.0)
        code = v.float().to(torch.float8_e4m3fn).view(torch.uint8).view(n, 512)
        return torch.cat((code, scale.view(torch.uint8).view(n, 16), tail), 1)
    g = x.view(n, 16, 32)
    most = g.abs().amax(2)
    e = torch.where(most > 0, (torch.frexp(most).exponent - 3).double(), torch.full_like(most, -127.0)).clamp(min=-127)
    v = groups_to_nearest(g * torch.exp2(-e)[..., None], 1, 0, 6.0)
    code = (v.abs()[..., None] == E2M1.to(v.device)).to(torch.int64).argmax(-1) + 8 * torch.signbit(g).long()
    code = code.view(n, 256, 2)
    return torch.cat(((code[..., 0] + 16 * code[..., 1]).to(torch.uint8), (e + 127).to(torch.uint8), tail), 1)


def unpack(rows, fmt):
    """uint8 rows [..., bytes] -> fp64 [..., 576]."""
    lead = rows.shape[:-1]
    rows = rows.contiguous().view(-1, BYTES[fmt])
    n = rows.shape[0]
    rope = rows[:, -128:].contiguous().view(torch.bfloat16).double()
    if fmt == 0:
        x = rows[:, :1024].contiguous().view(torch.bfloat16).double()
    elif fmt == 1:
        scale = rows[:, 512:528].contiguous().view(torch.float32).double()
        x = (rows[:, :512].contiguous().view(torch.float8_e4m3fn).double().view(n, 4, 128) * scale[..., None]).view(n, 512)
    else:
        b = rows[:, :256].long()
        nibble = torch.stack((b & 15, b >> 4), 2).view(n, 16, 32)
        v = E2M1.to(rows.device)[nibble & 7] * (1 - 2 * (nibble >> 3)).double()
        e = rows[:, 256:272].double()
        scale = torch.where(e == 255, torch.full_like(e, math.nan), torch.exp2(e - 127))
        x = (v * scale[..., None]).view(n, 512)
    return torch.cat((x, rope), 1).view(*lead, LATENT + ROPE)


def turn(x, positions, inv_freq, scale=1.0, halves=False):
    """fp64 [..., 64] turned by positions [...]."""
    angle = positions.double()[..., None] * torch.tensor(inv_freq, dtype=torch.float64, device=x.device)
    c, s = angle.cos() * scale, angle.sin() * scale
    x = x.double()
    out = torch.empty_like(x)
    first, second = (slice(0, 32), slice(32, 64)) if halves else (slice(0, None, 2), slice(1, None, 2))
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * c - b * s, a * s + b * c
    return out


def attend(q, buffer, slots, fmt, scale, softcap=0.0, ids=None, positions=None, spans=None, slopes=None, inv_freq=None, rope_scale=1.0, halves=False):
    """(out, lse, bound on |out|'s error, bound on lse's error), all fp64.

    The bounds.  A score is a sum of 576 products of bf16 queries with keys, added in 32 bits (576 x 2^-24 of the magnitudes' sum, doubled
    for the order of the matrix unit's adders and its cut-off bits), then a few operations of 2^-22 each on numbers up to the largest
    score or cap.  Queries may be two e4m3 numbers, of 4 bits each: off by 2^-17 of the largest one where an element is below 2^-10 of that; or fp16
    in units of 2^-14 of the largest number or finer (off by 2^-38 of it), with 4-bit rows in units of 2^-13 of the row's largest scale, elements
    off by 2^-25 of these.  d bounds the sum of these.  Weights then are off by a factor of exp(+-2 d) and rounded to 16 bits (bf16: 2^-8; fp16
    rows: three times 2^-11, the row's unit going onto them too); as fp16 they are whole to 2^-25 of 8 times the unit of the largest row (twice its
    scale) where the largest weight is 1 or more.  Values of 8-bit rows are fp16, in units of up to 2^-6 of the row's largest scale: off by 2^-11,
    twice (scale and product), and by 2^-25 x 448 of these units where a scale is far below the row's largest.  The result is rounded to bf16 (2^-8).  What is below 2^-126 may count as zero (weights next to the
    largest, results), and so may what is below 2^-100 in rows of 8 and 4 bits."""
    n, T, H, _ = q.shape
    dev = q.device
    outs, lses, eo, el = [], [], [], []
    for i in range(n):
        for g in range(T):
            s = slots[i, g].long()
            keep = (s >= 0) & (s < buffer.shape[1])
            if spans is not None:
                keep &= (ids[i, g] >= spans[i, g, 0]) & (ids[i, g] < spans[i, g, 1])
            at = torch.nonzero(keep).flatten()
            if at.numel() == 0:
                outs.append(torch.zeros(H, LATENT, dtype=torch.float64, device=dev)); lses.append(torch.full((H,), -math.inf, dtype=torch.float64, device=dev))
                eo.append(torch.zeros(H, LATENT, dtype=torch.float64, device=dev)); el.append(torch.zeros(H, dtype=torch.float64, device=dev))
                continue
            k = unpack(buffer[i, s[at]], fmt)
            x = q[i, g].double()
            if inv_freq is not None:
                x = torch.cat((x[:, :LATENT], turn(x[:, LATENT:], positions[i, g].expand(H), inv_freq, rope_scale, halves).to(torch.bfloat16).double()), 1)
            z = (x @ k.T) * scale
            size = (x.abs() @ k.abs().T) * abs(scale)
            d = size * (2 * 576 * 2.0 ** -24)
            fine = torch.zeros(at.numel(), dtype=torch.float64, device=dev)
            if fmt:
                raw = buffer[i, s[at]]
                if fmt == 1:
                    unit = raw[:, 512:528].contiguous().view(torch.float32).double().abs()
                    fine = 2.0 ** -25 * 448 * 2.0 ** -6 * unit.amax(1)
                else:
                    unit = torch.exp2(raw[:, 256:272].double().amax(1, keepdim=True).clamp(min=40) - 140)
                    fine = 2.0 ** -25 * unit[:, 0]
                spread = unit.repeat_interleave(512 // unit.shape[1], 1)
                top = x[:, :LATENT].abs().amax(1)[:, None]
                if fmt == 1:
                    d = d + abs(scale) * 2.0 ** -17 * (top * (x[:, :LATENT].abs() < top * 2.0 ** -9)) @ k[:, :LATENT].abs().T
                else:
                    d = d + abs(scale) * (2.0 ** -38 * top * k[:, :LATENT].abs().sum(1) + x[:, :LATENT].abs().sum(1)[:, None] * fine)
                code = torch.where(spread > 0, k[:, :LATENT].abs() / spread, torch.zeros_like(spread))
            if inv_freq is not None:        # a turned query that lies next to a border of bf16 may be rounded to its other side
                d = d + (x[:, LATENT:].abs() @ k[:, LATENT:].abs().T) * abs(scale) * 2.0 ** -7 * 0.02
            if softcap:
                z = softcap * torch.tanh(z / softcap)
                d = d + softcap * 2.0 ** -21
            if slopes is not None:
                away = (ids[i, g, at].long() - positions[i, g].long()).double()
                z = z + slopes.double()[:, None] * away
                d = d + (slopes.double()[:, None] * away).abs() * 2.0 ** -22
            d = (d + z.abs() * 2.0 ** -21).amax(1) + 2.0 ** -20
            lse = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[:, None])
            o, mass = p @ k[:, :LATENT], p @ k[:, :LATENT].abs()
            outs.append(o); lses.append(lse)
            less = mass * ((0.0, 5 * 2.0 ** -11, 3 * 2.0 ** -11)[fmt] + (0.0 if fmt else 2.0 ** -8) + torch.expm1(2 * d)[:, None]) + (p @ fine)[:, None]
            less = less + at.numel() * (2.0 ** -126 * k.abs().max() + (2.0 ** -100 if fmt else 0.0))
            if fmt:
                less = less + 2.0 ** -25 * 16 * unit.max() * code.sum(0) / torch.exp(lse - z.amax(1))[:, None]
            eo.append(less + (o.abs() + less) * 2.0 ** -8 + 2.0 ** -126); el.append(d + lse.abs() * 2.0 ** -22)
    back = lambda v, *tail: torch.stack(v).view(n, T, H, *tail)  # noqa: E731
    return back(outs, LATENT), back(lses), back(eo, LATENT), back(el)


def agree(out, lse, reference):
    want, want_lse, eo, el = reference
    off = (out.double() - want).abs()
    worst = (off - eo).max()
    assert bool((off <= eo).all()), "outputs are off by up to %.3g beyond their bound" % worst.item()
    if lse is not None:
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isneginf(lse), empty)
        assert bool(((lse.double() - want_lse).abs()[~empty] <= el[~empty]).all()), \
            "lse off by %.3g, allowed %.3g" % ((lse.double() - want_lse).abs()[~empty].max().item(), el[~empty].max().item())
