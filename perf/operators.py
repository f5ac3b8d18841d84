"""Operators beside the gather: rows appended to a cache, and the sparse attention that reads a slot table.

A row is what one position of a layer leaves in the cache: a latent of 512 numbers (keys and values at once) and 64 numbers
that carry the position's rotation.  It is held in one of three forms:
  bf16  1152 bytes: 512 + 64 bf16
  fp8    656 bytes: 512 e4m3, 4 fp32 scales (one for 128 numbers: largest magnitude / 448), 64 bf16
  fp4    400 bytes: 512 e2m1 (two to a byte, the even one in the low half), 16 e8m0 scales (one power of two for 32 numbers),
                    64 bf16
Sizes are those of the configurations and tests around the gather: top-K 256 to 2048 (1000 and odd ones too), 1 to 64 requests,
1 to 4 tokens of a multi-token prediction, 1024 to 8192 slots; 1 to 128 heads that share the row.

Keys of a case: op (attend, append), form, tables, tokens; attend: heads, topk, slots, ragged (selections of unequal length,
padded with -1), rotate (queries come without their rotation), shaped (scores capped by a tanh, a bias by distance, a document's
range of positions per query); append: rows (positions the cache has room for), first (the first position appended),
sliced (the rotated part is a slice of a wider projection), values (what the rows stand for is wanted too).
"""
import math
import random

import torch

own = False

LATENT, ROPE = 512, 64
ROW = {"bf16": 1152, "fp8": 656, "fp4": 400}
SHARED = 0.75                  # share of a token's selection that the table's first token has selected too
SCALE = 1.0 / math.sqrt(192.0)
CAP, BASE = 30.0, 10000.0
FP8_MOST, FP8_TINY = 448.0, 2.0 ** -126
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _attend(name, **kw):
    c = dict(op="attend", form="fp8", tables=1, tokens=1, heads=16, topk=2048, slots=8192, ragged=False, rotate=False, shaped=False)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def _append(name, **kw):
    c = dict(op="append", form="fp8", tables=1, tokens=1, rows=8192, first=0, sliced=False, values=False)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest configuration's selection, on one GPU of several that share the heads: all latency
        _attend("attend_one_short", topk=256, slots=1024),
        # one interactive request with token prediction and all heads, rows as the model computes them
        _attend("attend_one_bf16", form="bf16", tokens=2, heads=128),
        # the batch-32 configuration with all heads on the GPU: the most arithmetic
        _attend("attend_batch32", tables=32, tokens=2, heads=128),
        # the same batch where heads are shared among GPUs, rows in 4 bits: the link carries the least
        _attend("attend_batch32_fp4", form="fp4", tables=32, tokens=2, heads=16),
        # many unequal requests, the short ones selecting all that they have
        _attend("attend_unequal64", form="fp4", tables=64, heads=64, ragged=True),
        # an odd share of the heads, K not a power of two, queries as the projection leaves them
        _attend("attend_odd_heads", form="bf16", tables=8, heads=40, topk=1000, slots=4096, rotate=True),
        # packed documents with capped scores and a bias by distance, three predicted tokens
        _attend("attend_shaped", tables=16, tokens=4, heads=24, topk=2047, rotate=True, shaped=True),
        # one request's decode step
        _append("append_one", first=4095),
        # a batch's decode step with token prediction
        _append("append_batch64", tables=64, tokens=2, rows=2048, first=1000, sliced=True),
        # a prompt's chunk of four requests, whose own attention reads what the cache holds
        _append("append_chunk_fp4", form="fp4", tables=4, tokens=2048, rows=4096, first=1024, values=True),
        # a long prompt's chunk of odd length at far positions is held as it is
        _append("append_chunk_bf16", form="bf16", tokens=8191, rows=16384, first=8001, sliced=True),
        # a long prompt in 8 bits: the largest append
        _append("append_prompt", tables=2, tokens=16384, rows=16384, sliced=True),
    ]


def _spread(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def draw(rng):
    form = rng.choice(("bf16", "fp8", "fp4"))
    if rng.random() < 0.6:
        tokens = rng.choice((1, 1, 2, 2, 3, 4))
        topk = _spread(rng, 1, 2048)
        slots = 1 << max(5, (tokens * topk - 1).bit_length() + rng.choice((0, 1)))
        heads = rng.choice((1, 8, 16, 24, 32, 40, 64, 100, 128, rng.randint(1, 128)))
        tables = _spread(rng, 1, 64)
        while tables * tokens * topk > 32 * 2 * 2048:
            tables = (tables + 1) // 2
        return _attend("", form=form, tables=tables, tokens=tokens, heads=heads, topk=topk, slots=min(8192, slots), ragged=rng.random() < 0.3,
                       rotate=rng.random() < 0.4, shaped=rng.random() < 0.3)
    tables = _spread(rng, 1, 64)
    tokens = _spread(rng, 1, 16384)
    while tables * tokens > 32768:
        tables = (tables + 1) // 2
    first = rng.randint(0, 4096)
    return _append("", form=form, tables=tables, tokens=tokens, rows=first + tokens + rng.randint(0, 64), first=first, sliced=rng.random() < 0.5,
                   values=form == "fp4" or rng.random() < 0.5)


def _lengths(case):
    """How many ids each table's selections hold: by the case alone."""
    if not case["ragged"]:
        return [case["topk"]] * case["tables"]
    r = random.Random(case["topk"] * 1000 + case["tables"])
    return [_spread(r, 1, case["topk"]) for _ in range(case["tables"])]


# ---- what a program has in hand -----------------------------------------------------------------------------------

def _random_rows(shape, form, gen, dev):
    """Rows of random positions in their packed form (as a cache that has been filled holds them)."""
    n = 1
    for s in shape:
        n *= s
    out = torch.empty(n, ROW[form], dtype=torch.uint8, device=dev)
    size = torch.exp(0.4 * torch.randn(n, 1, generator=gen, device=dev))          # rows differ in magnitude
    x = torch.randn(n, LATENT, generator=gen, device=dev).mul_(size)
    r = torch.randn(n, ROPE, generator=gen, device=dev).to(torch.bfloat16).view(torch.uint8)
    if form == "bf16":
        out[:, :1024] = x.to(torch.bfloat16).view(torch.uint8)
        out[:, 1024:] = r
    elif form == "fp8":
        t = x.view(n, 4, 128)
        s = t.abs().amax(2) / FP8_MOST
        out[:, :512] = (t / s[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(n, 512)
        out[:, 512:528] = s.view(torch.uint8)
        out[:, 528:] = r
    else:
        codes = torch.randint(0, 256, (n, 256), generator=gen, device=dev, dtype=torch.uint8)
        out[:, :256] = codes
        out[:, 256:272] = (torch.log2(size) + 126).round().to(torch.uint8)
        out[:, 272:] = r
    return out.view(*shape, ROW[form])


def _prepare_attend(case, gen, dev):
    n, T, H, K, S = (case[k] for k in ("tables", "tokens", "heads", "topk", "slots"))
    s = {"buffer": _random_rows((n, S), case["form"], gen, dev)}
    q = torch.randn(n, T, H, LATENT + ROPE, generator=gen, device=dev)
    s["q"] = (q * (0.5 + torch.rand(n, T, H, 1, generator=gen, device=dev))).to(torch.bfloat16)
    # Selections: the slots of a table in random order; later tokens share most of the first one's.
    order = torch.rand(n, S, generator=gen, device=dev).argsort(1).to(torch.int32)
    shared = int(SHARED * K)
    slots = torch.empty(n, T, K, dtype=torch.int32, device=dev)
    slots[:, 0] = order[:, :K]
    for g in range(1, T):
        at = K + (g - 1) * (K - shared)
        slots[:, g, :shared] = order[:, :shared]
        slots[:, g, shared:] = order[:, at:at + K - shared]
    if case["ragged"]:
        length = torch.tensor(_lengths(case), device=dev)
        slots.masked_fill_(torch.arange(K, device=dev) >= length[:, None, None], -1)
    s["slots"] = slots
    s["positions"] = s["ids"] = s["spans"] = s["slopes"] = None
    if case["rotate"] or case["shaped"]:
        far = 1 << 17
        s["positions"] = (far + torch.arange(T, device=dev, dtype=torch.int32)).expand(n, T).contiguous()
    if case["shaped"]:
        # each slot holds some position; half of a selection is near the query, half anywhere in its context
        near = torch.rand(n, S, generator=gen, device=dev) < 0.5
        back = torch.rand(n, S, generator=gen, device=dev)
        held = torch.where(near, far - 1 - back * 4095, far - 1 - back * (far - 1)).to(torch.int32)
        s["ids"] = held.gather(1, slots.clamp(min=0).view(n, T * K).long()).view(n, T, K).masked_fill_(slots < 0, -1)
        begin = (torch.rand(n, T, generator=gen, device=dev) * (far // 2)).to(torch.int32)
        s["spans"] = torch.stack((begin, s["positions"] + 1), 2).contiguous()
        s["slopes"] = torch.exp2(-8.0 * (1 + torch.arange(H, device=dev, dtype=torch.float32)) / H) * 0.01
    s["inv_freq"] = [BASE ** (-i / 32.0) for i in range(32)] if case["rotate"] else None
    return s


def _prepare_append(case, gen, dev):
    n, T = case["tables"], case["tokens"]
    s = {"latent": torch.randn(n, T, LATENT, generator=gen, device=dev).to(torch.bfloat16)}
    if case["sliced"]:
        s["rope"] = torch.randn(n, T, LATENT + ROPE, generator=gen, device=dev).to(torch.bfloat16)[..., LATENT:]
    else:
        s["rope"] = torch.randn(n, T, ROPE, generator=gen, device=dev).to(torch.bfloat16)
    s["positions"] = (case["first"] + torch.arange(T, device=dev, dtype=torch.int32)).expand(n, T).contiguous()
    s["cache"] = torch.full((n, case["rows"], ROW[case["form"]]), 17, dtype=torch.uint8, device=dev)
    s["inv_freq"] = [BASE ** (-i / 32.0) for i in range(32)]
    return s


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    s = (_prepare_attend if case["op"] == "attend" else _prepare_append)(case, gen, dev)
    s["case"] = dict(case)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(s):
    attend = s["case"]["op"] == "attend"
    if own:
        return _own_attend(s) if attend else _own_append(s)
    return _plain_attend(s) if attend else _plain_append(s)


def _own_attend(s):
    import paper_2609_37538_b200 as avsg
    c = s["case"]
    rope = avsg.Rope(s["inv_freq"]) if c["rotate"] else None
    out, lse = avsg.attend(s["q"], s["buffer"], s["slots"], row_format=_format(avsg, c["form"]), scale=SCALE, want_lse=True, rope=rope,
                           positions=s["positions"], ids=s["ids"], spans=s["spans"], slopes=s["slopes"], softcap=CAP if c["shaped"] else 0.0)
    return out, lse


def _own_append(s):
    import paper_2609_37538_b200 as avsg
    c = s["case"]
    values = avsg.append(s["latent"], s["rope"], s["positions"], s["cache"], row_format=_format(avsg, c["form"]), rope=avsg.Rope(s["inv_freq"]),
                         want_values=c["values"])
    return _held(s["cache"], c["form"]) + ([values] if c["values"] else [])


def _format(avsg, form):
    return {"bf16": avsg.ROW_BF16, "fp8": avsg.ROW_FP8, "fp4": avsg.ROW_FP4}[form]


def _held(cache, form):
    """What the rows hold, as views of them."""
    if form == "bf16":
        return [cache.view(torch.bfloat16)]
    if form == "fp8":
        return [cache[..., :512].view(torch.float8_e4m3fn), cache[..., 512:528].view(torch.float32), cache[..., 528:].view(torch.bfloat16)]
    return [cache[..., :256], cache[..., 256:272], cache[..., 272:].view(torch.bfloat16)]


# The plain forms.

def _rows_to_float(rows, form):
    """[..., row bytes] -> [..., 576] in fp32."""
    if form == "bf16":
        return rows.view(torch.bfloat16).float()
    lead = rows.shape[:-1]
    if form == "fp8":
        x = rows[..., :512].contiguous().view(torch.float8_e4m3fn).float().view(*lead, 4, 128)
        x = x * rows[..., 512:528].contiguous().view(torch.float32)[..., None]
    else:
        b = rows[..., :256].int()
        table = torch.tensor(FP4 + tuple(-v for v in FP4), device=rows.device)
        x = torch.stack((table[b & 15], table[b >> 4]), -1).view(*lead, 16, 32)
        x = torch.ldexp(x, rows[..., 256:272].int()[..., None] - 127)
    return torch.cat((x.view(*lead, 512), rows[..., -128:].contiguous().view(torch.bfloat16).float()), -1)


def _rotated(x, positions, inv_freq):
    """Pairs (2i, 2i + 1) of the last 64 numbers turned by position * inv_freq[i]; angles in 64 bits."""
    angle = positions.double()[..., None] * torch.tensor(inv_freq, dtype=torch.float64, device=x.device)
    c, s = angle.cos().float(), angle.sin().float()
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)


def _plain_attend(s):
    c = s["case"]
    n, T, K = s["slots"].shape
    slots = s["slots"].long()
    q = s["q"].float()
    if c["rotate"]:
        q = torch.cat((q[..., :LATENT], _rotated(q[..., LATENT:], s["positions"][:, :, None], s["inv_freq"]).to(torch.bfloat16).float()), -1)
    table = torch.arange(n, device=slots.device)[:, None, None]
    k = _rows_to_float(s["buffer"][table, slots.clamp(min=0)], c["form"])
    score = torch.matmul(q, k.transpose(2, 3)) * SCALE
    keep = slots >= 0
    if c["shaped"]:
        score = CAP * torch.tanh(score / CAP)
        away = (s["positions"][:, :, None] - s["ids"]).float()
        score = score - s["slopes"][:, None] * away[:, :, None, :]
        keep = keep & (s["ids"] >= s["spans"][:, :, :1]) & (s["ids"] < s["spans"][:, :, 1:])
    score = score.masked_fill(~keep[:, :, None, :], -math.inf)
    most = score.amax(3, keepdim=True)
    p = torch.where(keep[:, :, None, :], torch.exp(score - most), torch.zeros_like(score))
    total = p.sum(3, keepdim=True)
    out = torch.where(total > 0, torch.matmul(p, k[..., :LATENT]) / total, torch.zeros_like(total))
    return out.to(torch.bfloat16), (most + torch.log(total)).squeeze(3)


def _plain_append(s):
    c = s["case"]
    x, form = s["latent"].float(), c["form"]
    n, T, _ = x.shape
    turned = _rotated(s["rope"].float(), s["positions"], s["inv_freq"]).to(torch.bfloat16)
    if form == "bf16":
        parts, stands = [s["latent"].view(torch.uint8)], x
    elif form == "fp8":
        t = x.view(n, T, 4, 128)
        scale = (t.abs().amax(3) / torch.tensor(FP8_MOST, device=x.device)).clamp(min=FP8_TINY)       # (by a number: times its reciprocal)
        code = (t / scale[..., None]).clamp(-FP8_MOST, FP8_MOST).to(torch.float8_e4m3fn)
        parts = [code.view(n, T, 512).view(torch.uint8), scale.view(torch.uint8)]
        stands = code.float() * scale[..., None]
    else:
        t = x.view(n, T, 16, 32)
        most = t.abs().amax(3)
        e = torch.where(most > 0, torch.frexp(most).exponent - 3, torch.full_like(most, -127, dtype=torch.int32)).clamp(-127, 127)
        size = torch.ldexp(t.abs(), -e[..., None])
        # to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6; of two as near the one with the even code
        code = (size > 0.25).int() + (size >= 0.75).int() + (size > 1.25).int() + (size >= 1.75).int() + (size > 2.5).int() + (size >= 3.5).int() + (size > 5.0).int()
        sign = t.signbit().int() * 8
        b = (code + sign).view(n, T, 256, 2)
        parts = [(b[..., 0] + 16 * b[..., 1]).to(torch.uint8), (e + 127).to(torch.uint8)]
        mag = torch.tensor(FP4, device=x.device)[code]
        stands = torch.ldexp(torch.where(sign > 0, -mag, mag), e[..., None])
    rows = torch.cat(parts + [turned.view(torch.uint8)], -1)
    s["cache"][torch.arange(n, device=x.device)[:, None], s["positions"].long()] = rows
    out = _held(s["cache"], form)
    return out + ([torch.cat((stands.reshape(n, T, 512).to(torch.bfloat16), turned), -1)] if c["values"] else [])


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    if case["op"] == "append":
        n = case["tables"] * case["tokens"]
        return {"bytes": n * (1152 + 4 + ROW[case["form"]] + (1152 if case["values"] else 0)), "flops": n * (512 * 3 + 64 * 3)}
    T, H, K = case["tokens"], case["heads"], case["topk"]
    total = flops = 0
    for length in _lengths(case):
        shared = min(int(SHARED * K), length)
        total += (length + (T - 1) * (length - shared)) * ROW[case["form"]]
        flops += T * H * length * 2 * (LATENT + ROPE + LATENT)
        total += T * length * (8 if case["shaped"] else 4) + T * H * (1152 + 1024 + 4)
    return {"bytes": total, "flops": flops}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attend(s)


def _turn64(x, pos, inv_freq):
    z = torch.view_as_complex(x.double().reshape(*x.shape[:-1], 32, 2).contiguous())
    w = torch.polar(torch.ones(32, dtype=torch.float64, device=x.device), torch.zeros(32, dtype=torch.float64, device=x.device))
    f = torch.tensor(inv_freq, dtype=torch.float64, device=x.device)
    w = w * torch.exp(1j * (pos.double().unsqueeze(-1) * f))
    return torch.view_as_real(z * w).reshape(x.shape)


def _row64(rows, form):
    """Packed rows -> [..., 576] in 64 bits, number by number from the formats' definitions."""
    def bf(two):
        w = two.reshape(*two.shape[:-1], -1, 2).to(torch.int64)
        w = w[..., 0] + 256 * w[..., 1]
        e, m, neg = (w >> 7) & 255, w & 127, w >> 15
        v = torch.where(e > 0, torch.ldexp(1 + m.double() / 128, (e - 127)), torch.ldexp(m.double() / 128, torch.full_like(e, -126)))
        return torch.where(neg > 0, -v, v)
    if form == "bf16":
        return bf(rows)
    if form == "fp8":
        b = rows[..., :512].to(torch.int64)
        e, m = (b >> 3) & 15, b & 7
        v = torch.where(e > 0, torch.ldexp(1 + m.double() / 8, e - 7), m.double() * 2.0 ** -9)
        v = torch.where(b > 127, -v, v)
        sc = rows[..., 512:528].contiguous().view(torch.float32).double().repeat_interleave(128, -1)
    else:
        b = rows[..., :256].to(torch.int64)
        nib = torch.stack((b % 16, b // 16), -1).flatten(-2)
        e, m = (nib >> 1) & 3, nib & 1
        v = torch.where(e > 0, torch.ldexp(1 + m.double() / 2, e - 1), m.double() / 2)
        v = torch.where(nib > 7, -v, v)
        sc = torch.ldexp(torch.ones((), dtype=torch.float64, device=rows.device), rows[..., 256:272].to(torch.int64) - 127).repeat_interleave(32, -1)
    return torch.cat((v * sc, bf(rows[..., -128:])), -1)


def _exact_attend(s):
    c = s["case"]
    n, T, H, _ = s["q"].shape
    outs, lses = [], []
    for i in range(n):
        for g in range(T):
            at = torch.nonzero(s["slots"][i, g] >= 0).flatten()
            if c["shaped"]:
                x = s["ids"][i, g, at]
                at = at[(x >= s["spans"][i, g, 0]) & (x < s["spans"][i, g, 1])]
            if at.numel() == 0:
                outs.append(torch.zeros(H, LATENT, dtype=torch.float64, device=at.device))
                lses.append(torch.full((H,), -math.inf, dtype=torch.float64, device=at.device))
                continue
            rows = _row64(s["buffer"][i, s["slots"][i, g, at].long()], c["form"])
            q = s["q"][i, g].double()
            if c["rotate"]:
                turned = _turn64(q[:, LATENT:], s["positions"][i, g].expand(H), s["inv_freq"])
                q = torch.cat((q[:, :LATENT], turned.to(torch.bfloat16).double()), 1)     # (a turned query is a bf16 query again)
            z = (q @ rows.T) * SCALE
            if c["shaped"]:
                z = CAP * torch.tanh(z / CAP) + s["slopes"].double()[:, None] * (s["ids"][i, g, at] - s["positions"][i, g]).double()
            lse = torch.logsumexp(z, 1)
            outs.append(torch.exp(z - lse[:, None]) @ rows[:, :LATENT])
            lses.append(lse)
    return torch.stack(outs).view(n, T, H, LATENT), torch.stack(lses).view(n, T, H)


def _nearest64(x, mantissa, least):
    """x to the nearest number with so many bits behind the leading one, steps no finer than at 2 ** least; ties to even."""
    e = (torch.frexp(x).exponent - 1).clamp(min=least)
    step = torch.ldexp(torch.ones_like(x), e - mantissa)
    return torch.round(x / step) * step


def _exact_append(s):
    c = s["case"]
    x = s["latent"].double()
    n, T, _ = x.shape
    R = c["rows"]
    turned = _turn64(s["rope"], s["positions"], s["inv_freq"])
    at = (torch.arange(n, device=x.device)[:, None], s["positions"].long())
    old = _held(s["cache"], c["form"])

    def placed(k, rows):
        whole = old[k].to(rows.dtype).clone()
        whole[at] = rows
        return whole

    if c["form"] == "bf16":
        out, stands = [placed(0, torch.cat((x, turned), -1))], x
    elif c["form"] == "fp8":
        t = x.view(n, T, 4, 128)
        scale = (t.abs().amax(3) / FP8_MOST).float().clamp(min=FP8_TINY).double()
        v = _nearest64(t / scale[..., None], 3, -6).clamp(-448, 448)
        out = [placed(0, v.view(n, T, 512)), placed(1, scale), placed(2, turned)]
        stands = (v * scale[..., None]).view(n, T, 512)
    else:
        t = x.view(n, T, 16, 32)
        e = torch.floor(torch.log2(t.abs().amax(3))).clamp(min=-125) - 2
        v = _nearest64(t / torch.exp2(e)[..., None], 1, 0).clamp(-6, 6)
        half = (v.abs() * 2).round().long()
        code = torch.tensor([0, 1, 2, 3, 4, 4, 5, 5, 6, 6, 6, 6, 7], device=x.device)[half] + 8 * torch.signbit(t).long()
        b = code.view(n, T, 256, 2)
        out = [placed(0, (b[..., 0] + 16 * b[..., 1]).to(torch.uint8)), placed(1, (e + 127).to(torch.uint8)), placed(2, turned)]
        stands = (v * torch.exp2(e)[..., None]).view(n, T, 512)
    return out + ([torch.cat((stands, turned), -1)] if c["values"] else [])
