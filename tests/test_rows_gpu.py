"""avsg_append and avsg_attend against their definitions in 64 bits, on a B200."""
import math

import pytest

pytestmark = pytest.mark.gpu

FORMATS = [0, 1, 2]
INV_FREQ = [10000.0 ** (-i / 32) for i in range(32)]


@pytest.fixture(scope="module")
def avsg():
    import torch
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2609_37538_b200 as m
    m.load_library()
    return m


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _problem(fmt, n, T, H, K, S, seed=0, spread=0.5):
    import torch
    import rows_reference as ref
    g = _gen(seed)
    buffer = ref.random_rows((n, S), fmt, g, "cuda", spread)
    q = (torch.randn(n, T, H, 576, generator=g, device="cuda") * (0.5 + torch.rand(n, T, H, 1, generator=g, device="cuda"))).to(torch.bfloat16)
    slots = torch.stack([torch.stack([torch.randperm(S, generator=g, device="cuda")[:K] if K <= S else
                                      torch.randint(0, S, (K,), generator=g, device="cuda") for _ in range(T)]) for _ in range(n)]).to(torch.int32)
    return q, buffer, slots


SCALE = 192 ** -0.5


# ---- attention ---------------------------------------------------------------------------------------------------
SIZES = [
    # n, tokens, heads, topk, slots
    (1, 1, 1, 1, 32),
    (1, 1, 16, 2, 32),
    (2, 3, 5, 37, 128),
    (1, 1, 16, 256, 1024),
    (3, 2, 64, 64, 256),
    (2, 1, 65, 65, 128),
    (1, 2, 128, 130, 256),
    (2, 1, 100, 1000, 4096),
    (1, 1, 17, 2049, 4096),
    (1, 4, 24, 2048, 8192),
    (5, 1, 33, 191, 512),
    (40, 2, 8, 129, 512),       # more queries than half of the SMs
    (90, 2, 72, 70, 256),       # more than all of them
    (1, 1, 300, 100, 128),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_attend(avsg, fmt, size):
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, *size, seed=sum(size))
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True)
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, SCALE))


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_padding_anywhere(avsg, fmt):
    # nothing selected; only the first or the last; whole stretches of 64 and 128 empty in front, between and behind; single holes
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 8, 1, 20, 400, 512, seed=3)
    slots[0] = -1
    slots[1, :, 1:] = -1
    slots[2, :, :-1] = -1
    slots[3, :, :200] = -1
    slots[4, :, 64:192] = -1
    slots[5, :, 130:] = -1
    slots[6, :, ::2] = -1
    slots[7, :, 255:257] = -7
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True)
    assert not out[0].any() and torch.isneginf(lse[0]).all()
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, SCALE))


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_the_same_row_many_times(avsg, fmt):
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 1, 2, 16, 300, 32, seed=4)
    slots[0, 0] = 5
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True)
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, SCALE))


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_does_not_read_what_is_masked(avsg, fmt):
    # rows that no query may see hold NaN and infinity; some are not selected, some are outside of the spans
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 2, 2, 9, 150, 256, seed=5)
    ids = slots * 3
    spans = torch.tensor([[[0, 300], [150, 768]], [[600, 768], [0, 0]]], dtype=torch.int32, device="cuda")
    poison = buffer.clone()
    seen = torch.zeros(2, 256, dtype=torch.bool, device="cuda")
    for i in range(2):
        for g in range(2):
            ok = (ids[i, g] >= spans[i, g, 0]) & (ids[i, g] < spans[i, g, 1])
            seen[i, slots[i, g][ok].long()] = True
    poison[~seen] = 255
    a = avsg.attend(q, poison, slots, row_format=fmt, scale=SCALE, want_lse=True, ids=ids, spans=spans)
    assert not a[0][1, 1].any() and torch.isneginf(a[1][1, 1]).all()
    ref.agree(*a, ref.attend(q, buffer, slots, fmt, SCALE, ids=ids, spans=spans))


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_nan_in_a_seen_row_reaches_only_its_queries(avsg, fmt):
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 2, 1, 16, 100, 256, seed=6)
    bad = buffer.clone()
    at = slots[1, 0, 70].item()
    if fmt == 0:
        bad[1, at, :2] = torch.tensor([0xC0, 0x7F], dtype=torch.uint8)
    elif fmt == 1:
        bad[1, at, 3] = 0x7F
    else:
        bad[1, at, 256 + 5] = 255
    out, lse = avsg.attend(q, bad, slots, row_format=fmt, scale=SCALE, want_lse=True)
    assert torch.isnan(lse[1]).all() and torch.isnan(out[1]).any()
    want = ref.attend(q, buffer, slots, fmt, SCALE)
    ref.agree(out[:1], lse[:1], tuple(w[:1] for w in want))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("size", [(2, 3, 16, 100, 512), (1, 1, 70, 513, 1024)], ids=lambda s: "x".join(map(str, s)))
def test_attend_shaped_scores(avsg, fmt, halves, size):
    # capped, with a bias by distance, masked by spans, queries rotated at positions around 2^20
    import torch
    import rows_reference as ref
    n, T, H, K, S = size
    q, buffer, slots = _problem(fmt, *size, seed=7)
    slots[0, 0, ::5] = -1
    g = _gen(8)
    positions = (1 << 20) + torch.arange(n * T, device="cuda", dtype=torch.int32).view(n, T)
    ids = torch.randint(0, 1 << 20, (n, T, K), generator=g, device="cuda", dtype=torch.int32)
    spans = torch.stack((torch.randint(0, 1 << 19, (n, T), generator=g, device="cuda", dtype=torch.int32), positions + 1), 2).contiguous()
    slopes = -torch.rand(H, generator=g, device="cuda") * 1e-5
    rope = avsg.Rope(INV_FREQ, 1.25, halves)
    kw = dict(softcap=15.0, ids=ids, positions=positions, spans=spans, slopes=slopes)
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True, rope=rope, **kw)
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, SCALE, inv_freq=INV_FREQ, rope_scale=1.25, halves=halves, **kw))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("one", ["softcap", "slopes", "spans", "rope"])
def test_attend_one_option_at_a_time(avsg, fmt, one):
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 2, 2, 12, 200, 256, seed=9)
    positions = torch.tensor([[0, 7], [300, 2000]], dtype=torch.int32, device="cuda")
    ids = slots + 4
    kw = {"softcap": dict(softcap=3.0), "slopes": dict(slopes=torch.linspace(-0.01, 0.02, 12, device="cuda"), ids=ids, positions=positions),
          "spans": dict(spans=torch.tensor([[[0, 100], [50, 51]], [[-5, 10], [4, 260]]], dtype=torch.int32, device="cuda"), ids=ids),
          "rope": dict(positions=positions)}[one]
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True, rope=avsg.Rope(INV_FREQ) if one == "rope" else None, **kw)
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, SCALE, inv_freq=INV_FREQ if one == "rope" else None, **kw))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size,rows", [(30.0, 0.0), (1e-20, 3.0), (1e18, 0.0)], ids=["peaked", "tiny", "huge"])
def test_attend_magnitudes(avsg, fmt, size, rows):
    # one position carries nearly all weight; queries far from one with a scale that brings the scores back; rows of very different sizes
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 2, 1, 18, 300, 512, seed=11, spread=max(rows, 0.5))
    q = (q.float() * size).to(torch.bfloat16)
    scale = SCALE if size == 30.0 else SCALE / size
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=scale, want_lse=True)
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, scale))


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_scores_that_rise_and_fall_along_the_list(avsg, fmt):
    # the running maximum moves in every stretch of positions, up to far beyond what was weighed before; and the other way round
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 2, 1, 40, 512, 512, seed=12)
    z = (q[:, 0].double() @ ref.unpack(buffer, fmt).transpose(1, 2))[:, 3]         # by head 3's scores
    order = z.argsort(1)
    slots[0, 0] = order[0].to(torch.int32)
    slots[1, 0] = order[1].flip(0).to(torch.int32)
    for scale in (SCALE, 20 * SCALE):
        out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=scale, want_lse=True)
        ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, scale))


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_rows_of_zeros_and_rising_sizes(avsg, fmt):
    # a row of zeros that takes nearly all weight by its rotated part; rows each twice the size of the one before
    import torch
    import rows_reference as ref
    g = _gen(13)
    x = torch.randn(256, 512, generator=g, device="cuda", dtype=torch.float64) * torch.exp2(torch.arange(256, device="cuda") / 16.0 - 8)[:, None]
    x[100] = 0
    r = torch.randn(256, 64, generator=g, device="cuda").to(torch.bfloat16)
    buffer = ref.pack(x, r, fmt)[None].contiguous()
    q = torch.zeros(1, 1, 4, 576, device="cuda", dtype=torch.bfloat16)
    q[0, 0, 0, 512:] = (r[100].float() * 4).to(torch.bfloat16)
    q[0, 0, 1:] = (torch.randn(3, 576, generator=g, device="cuda") * 0.01).to(torch.bfloat16)
    for slots in (torch.arange(256, device="cuda"), torch.arange(255, -1, -1, device="cuda")):
        slots = slots.to(torch.int32).view(1, 1, 256)
        out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True)
        ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, SCALE))


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_strides(avsg, fmt):
    # queries and outputs as slices of wider tensors, heads in front of tokens; a buffer with room behind its rows
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 2, 3, 10, 90, 128, seed=14)
    want = ref.attend(q, buffer, slots, fmt, SCALE)
    wide = torch.full((2, 10, 3, 640), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[..., 32:608] = q.transpose(1, 2)
    roomy = torch.full((2, 128, buffer.shape[2] + 48), 255, dtype=torch.uint8, device="cuda")
    roomy[..., :buffer.shape[2]] = buffer
    store = torch.full((2, 10, 3, 528), 3.0, dtype=torch.bfloat16, device="cuda")
    out = store[..., 8:520].transpose(1, 2)
    lse = torch.empty(2, 3, 10, device="cuda")
    got = avsg.attend(wide[..., 32:608].transpose(1, 2), roomy[..., :buffer.shape[2]], slots, row_format=fmt, scale=SCALE, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    ref.agree(out, lse, want)
    assert (store[..., :8] == 3.0).all() and (store[..., 520:] == 3.0).all()


def test_attend_bad_slots_are_masked_and_reported(avsg):
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(1, 2, 1, 16, 100, 128, seed=15)
    slots[0, 0, 10] = 128
    slots[1, 0, 99] = 2 ** 31 - 1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = avsg.attend(q, buffer, slots, row_format=1, scale=SCALE, want_lse=True, status=status)
    assert status.item() == avsg.STATUS_BAD_SLOT
    ref.agree(out, lse, ref.attend(q, buffer, slots, 1, SCALE))
    out2 = avsg.attend(q, buffer, slots, row_format=1, scale=SCALE)
    assert torch.equal(out, out2)


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_repeats_bit_for_bit(avsg, fmt):
    import torch
    q, buffer, slots = _problem(fmt, 3, 2, 48, 700, 1024, seed=16)
    first = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True)
    for _ in range(20):
        again = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_attend_streams_and_graphs(avsg):
    # two calls at once on two streams; a call captured, its inputs changed, and replayed, together with another graph
    import torch
    import rows_reference as ref
    a = _problem(1, 4, 2, 64, 500, 1024, seed=17)
    b = _problem(2, 3, 1, 16, 300, 512, seed=18)
    want_a, want_b = ref.attend(*a, 1, SCALE), ref.attend(*b, 2, SCALE)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(10):
        with torch.cuda.stream(s1):
            got.append((avsg.attend(*a, row_format=1, scale=SCALE, want_lse=True), want_a))
        with torch.cuda.stream(s2):
            got.append((avsg.attend(*b, row_format=2, scale=SCALE, want_lse=True), want_b))
    torch.cuda.synchronize()
    for g, w in got:
        ref.agree(*g, w)
    graphs = []
    for args, fmt in ((a, 1), (b, 2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, avsg.attend(*args, row_format=fmt, scale=SCALE, want_lse=True)))
    c = _problem(1, 4, 2, 64, 500, 1024, seed=19)
    for to, x in zip(a, c):
        to.copy_(x)
    want_a = ref.attend(*a, 1, SCALE)
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            graphs[0][0].replay()
        with torch.cuda.stream(s2):
            graphs[1][0].replay()
    torch.cuda.synchronize()
    ref.agree(*graphs[0][1], want_a)
    ref.agree(*graphs[1][1], want_b)


def test_attend_far_into_a_large_buffer(avsg):
    # tables and rows beyond 2^32 bytes
    import torch
    import rows_reference as ref
    q, small, slots = _problem(0, 2, 1, 8, 60, 64, seed=20)
    rows = 2_000_000
    buffer = torch.empty((2, rows, 1152), dtype=torch.uint8, device="cuda")
    buffer[0, rows - 64:] = small[0]
    buffer[1, rows - 64:] = small[1]
    out, lse = avsg.attend(q, buffer, slots + (rows - 64), row_format=0, scale=SCALE, want_lse=True)
    ref.agree(out, lse, ref.attend(q, small, slots, 0, SCALE))


def test_attend_many_tables(avsg):
    # more tables than the small argument block holds, through a context, in another order than they lie in
    import torch
    import rows_reference as ref
    n, S = 200, 32
    ctx = avsg.Context(num_tables=n, buffer_slots=S, row_bytes=400, max_topk=16)
    q, rows, slots = _problem(2, n, 1, 4, 16, S, seed=21)
    order = torch.randperm(n).tolist()
    for i, t in enumerate(order):
        ctx.buffer(t).copy_(rows[i])
    out, lse = ctx.attend(order, q, slots, row_format=avsg.ROW_FP4, scale=SCALE, want_lse=True)
    ref.agree(out, lse, ref.attend(q, rows, slots, 2, SCALE))
    slots[150, 0, 3] = S
    ctx.attend([7] * n, q, slots, row_format=avsg.ROW_FP4, scale=SCALE)
    assert ctx.sync_status() == avsg.STATUS_BAD_SLOT
    ctx.clear_status()
    for bad in (dict(row_format=avsg.ROW_FP8), dict(row_format=avsg.ROW_FP4, status=slots)):
        with pytest.raises(avsg.AvsgError):
            ctx.attend(order, q, slots, scale=SCALE, **bad)
    with pytest.raises(avsg.AvsgError):
        ctx.attend([n] * n, q, slots, row_format=avsg.ROW_FP4, scale=SCALE)


@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("size", [(3, 2, 20, 200, 256), (2, 1, 64, 700, 1024)], ids=lambda s: "x".join(map(str, s)))
def test_attend_scales_far_apart_within_a_row_and_between_rows(avsg, fmt, size):
    # 8 bits: groups of a row from 2^-20 to 2^4, some negative, some zero; 4 bits: groups 2^-18 .. 1 of each other; a few rows of 2^6 times the others' size
    import torch
    import rows_reference as ref
    n, T, H, K, S = size
    q, buffer, slots = _problem(fmt, *size, seed=61 + fmt)
    g = _gen(62 + fmt)
    rows = buffer.view(-1, buffer.shape[-1])
    large = torch.rand(rows.shape[0], 1, generator=g, device="cuda") < 0.02
    if fmt == 1:
        power = torch.randint(-26, -1, (rows.shape[0], 4), generator=g, device="cuda").double() + 6.0 * large
        scale = torch.exp2(power) * (1 + torch.rand(rows.shape[0], 4, generator=g, device="cuda"))
        scale *= torch.where(torch.rand(rows.shape[0], 4, generator=g, device="cuda") < 0.1, -1.0, 1.0)
        scale[torch.rand(rows.shape[0], 4, generator=g, device="cuda") < 0.1] = 0.0
        rows[:, 512:528] = scale.float().view(torch.uint8)
    else:
        code = torch.randint(105, 124, (rows.shape[0], 16), generator=g, device="cuda") + 6 * large
        code[torch.rand(rows.shape[0], 16, generator=g, device="cuda") < 0.05] = 0
        rows[:, 256:272] = code.to(torch.uint8)
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=0.01, want_lse=True)
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, 0.01))


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_a_table_that_stands_twice_in_a_call(avsg, fmt):
    # a context's tables may repeat: two blocks of queries read the same buffer
    import torch
    import rows_reference as ref
    rb = ref.BYTES[fmt]
    ctx = avsg.Context(num_tables=2, buffer_slots=128, row_bytes=rb, max_topk=32, max_tokens=1)
    try:
        q, buffer, slots = _problem(fmt, 3, 1, 18, 32, 128, seed=71)
        kv = [buffer[i].contiguous() for i in range(2)]
        ids = torch.stack([torch.randperm(128, generator=_gen(72), device="cuda")[:32] for _ in range(2)]).to(torch.int32).view(2, 1, 32)
        step = ctx.step([0, 1], ids, kv, [128, 128])
        at = step.slots[[1, 0, 1]].contiguous()
        got = ctx.attend([1, 0, 1], q, at, row_format=fmt, scale=SCALE, want_lse=True)
        held = torch.stack([kv[1], kv[0], kv[1]])
        ref.agree(*got, ref.attend(q, held, ids[[1, 0, 1]].contiguous(), fmt, SCALE))
        assert ctx.sync_status() == 0
    finally:
        ctx.close()


# ---- appending ------------------------------------------------------------------------------------------------------
def _rows_agree(got, want, fmt, turned):
    """Latent bytes are the definition's, bit for bit; the rotated part is a bf16 beside the exact one."""
    import torch
    body = got.shape[-1] - 128
    assert torch.equal(got[..., :body], want[..., :body]), "%d latent bytes differ" % int((got[..., :body] != want[..., :body]).sum())
    tail = got[..., body:].contiguous().view(torch.bfloat16).double()
    # fp32 products and sum before the rounding: 3 x 2^-24 of the pair's size, and the angle's cosine to 2^-22
    slack = 2.0 ** -20 * turned.abs().amax(-1, keepdim=True).clamp(min=1.0) * 2
    assert bool(((tail - turned).abs() <= turned.abs() * 2.0 ** -8 + slack).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("size", [(1, 1), (3, 2), (2, 129), (130, 1)], ids=lambda s: "x".join(map(str, s)))
def test_append(avsg, fmt, dtype, size):
    import torch
    import rows_reference as ref
    n, T = size
    dt = getattr(torch, dtype)
    g = _gen(30)
    latent = (torch.randn(n, T, 512, generator=g, device="cuda") * torch.exp(torch.randn(n, T, 1, generator=g, device="cuda"))).to(dt)
    part = torch.randn(n, T, 64, generator=g, device="cuda").to(dt)
    latent[0, 0, :128] = 0
    R = T + 60
    positions = torch.stack([torch.randperm(R, generator=g, device="cuda")[:T] for _ in range(n)]).to(torch.int32)
    if T > 1:
        positions[0, 1] = -1
    kv = torch.randint(0, 256, (n, R, ref.BYTES[fmt]), generator=g, device="cuda", dtype=torch.uint8)
    before = kv.clone()
    values = avsg.append(latent, part, positions, kv, row_format=fmt, rope=avsg.Rope(INV_FREQ, 0.75), want_values=True)
    turned = ref.turn(part, positions, INV_FREQ, 0.75)
    written = positions >= 0
    packed = ref.pack(latent.double().view(-1, 512), turned.to(torch.bfloat16).view(-1, 64), fmt).view(n, T, -1)
    at = (torch.arange(n, device="cuda")[:, None].expand(n, T)[written], positions[written].long())
    _rows_agree(kv[at], packed[written], fmt, turned[written])
    stands = ref.unpack(kv[at], fmt)
    assert torch.equal(values[written], stands.float().to(torch.bfloat16))
    kv[at] = before[at]
    assert torch.equal(kv, before), "rows that no token names were written"


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_ties_extremes_and_what_is_not_a_number(avsg, fmt):
    import torch
    import rows_reference as ref
    g = _gen(31)
    T = 12
    x = torch.zeros(T, 512, device="cuda")
    grid = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7], device="cuda")
    x[0] = grid.repeat(32) * torch.where(torch.arange(512, device="cuda") % 3 == 0, -1.0, 1.0)          # ties of e2m1
    x[1] = torch.arange(512, device="cuda") * 1.75 - 448                                                   # around ties of e4m3
    x[2] = 1e30 * torch.randn(512, generator=g, device="cuda")
    x[3] = 1e-30 * torch.randn(512, generator=g, device="cuda")
    x[4, 17] = 2.0 ** -120
    x[5] = torch.randn(512, generator=g, device="cuda")
    x[5, 3] = 3e38
    x[6] = -0.0
    x[7] = 448.0
    x[8:] = torch.randn(4, 512, generator=g, device="cuda") * torch.exp2(torch.arange(512, device="cuda") / 16 - 16)
    x = x.to(torch.bfloat16)[None]
    part = torch.zeros(1, T, 64, device="cuda", dtype=torch.bfloat16)
    positions = torch.arange(T, device="cuda", dtype=torch.int32)[None]
    kv = torch.zeros(1, T, ref.BYTES[fmt], dtype=torch.uint8, device="cuda")
    avsg.append(x, part, positions, kv, row_format=fmt)
    assert torch.equal(kv[0], ref.pack(x[0].double(), part[0], fmt))
    if fmt:
        # a group with an infinity or a NaN stands for NaN, and only that group
        y = x.clone()
        y[0, 8, 5], y[0, 9, 200], y[0, 10, 511] = math.nan, math.inf, -math.inf
        values = avsg.append(y, part, positions, kv, row_format=fmt, want_values=True)
        want = ref.unpack(ref.pack(x[0].double(), part[0], fmt), fmt)
        size = 128 if fmt == 1 else 32
        for t, d in ((8, 5), (9, 200), (10, 511)):
            want[t, d // size * size:(d // size + 1) * size] = math.nan
        got = ref.unpack(kv[0], fmt)
        assert torch.equal(torch.nan_to_num(got, nan=9e9), torch.nan_to_num(want, nan=9e9))
        assert torch.equal(torch.isnan(values[0]), torch.isnan(want))


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_far_positions_halves_and_slices(avsg, fmt):
    # positions up to 2^30 go to other rows; the rotated part and the latent are slices of one projection
    import torch
    import rows_reference as ref
    g = _gen(32)
    both = torch.randn(2, 5, 640, generator=g, device="cuda").to(torch.bfloat16)
    latent, part = both[..., 64:576], both[..., 576:]
    positions = torch.tensor([[0, 1, 131071, (1 << 20) + 3, (1 << 30) - 1]] * 2, dtype=torch.int32, device="cuda")
    rows = torch.tensor([[3, 0, -1, 7, 2], [9, 8, 11, 10, 12]], dtype=torch.int32, device="cuda")
    pool = torch.zeros(13, ref.BYTES[fmt], dtype=torch.uint8, device="cuda")           # one pool for both tables
    avsg.append(latent, part, positions, pool, row_format=fmt, rows=rows, rope=avsg.Rope(INV_FREQ, 1.0, halves=True))
    turned = ref.turn(part, positions, INV_FREQ, 1.0, True)
    keep = rows >= 0
    packed = ref.pack(latent.double().reshape(-1, 512), turned.to(torch.bfloat16).view(-1, 64), fmt).view(2, 5, -1)
    _rows_agree(pool[rows[keep].long()], packed[keep], fmt, turned[keep])
    assert not pool[[1, 4, 5, 6]].any()


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_reports_rows_beyond_the_cache(avsg, fmt):
    import torch
    import rows_reference as ref
    kv = torch.zeros(2, 4, ref.BYTES[fmt], dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    x, part = torch.ones(2, 2, 512, device="cuda"), torch.ones(2, 2, 64, device="cuda")
    avsg.append(x, part, torch.tensor([[0, 3], [4, 1]], dtype=torch.int32, device="cuda"), kv, row_format=fmt, status=status)
    assert status.item() == avsg.STATUS_BAD_ID
    assert (kv.any(-1) == torch.tensor([[1, 0, 0, 1], [0, 1, 0, 0]], dtype=torch.bool, device="cuda")).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_to_pinned_memory(avsg, fmt):
    import torch
    import rows_reference as ref
    g = _gen(33)
    n, T, R = 3, 2, 50
    rb = ref.BYTES[fmt]
    latent = torch.randn(n, T, 512, generator=g, device="cuda").to(torch.bfloat16)
    part = torch.randn(n, T, 64, generator=g, device="cuda").to(torch.bfloat16)
    positions = torch.tensor([[0, 49], [7, 8], [30, 2]], dtype=torch.int32, device="cuda")
    want = ref.pack(latent.double().view(-1, 512), part.view(-1, 64), fmt).view(n, T, rb).cpu()
    apart = [avsg.pinned_empty(R * (rb + 16)) for _ in range(n)]
    for k in apart:
        k.zero_()
    together = torch.zeros(n, R, rb, dtype=torch.uint8, pin_memory=True)
    avsg.append(latent, part, positions, apart, row_format=fmt, row_stride=[rb + 16] * n, kv_rows=[R] * n)
    avsg.append(latent, part, positions, together, row_format=fmt)
    torch.cuda.synchronize()
    for i in range(n):
        for t in range(T):
            r = positions[i, t].item()
            assert torch.equal(apart[i].view(R, rb + 16)[r, :rb], want[i, t]) and torch.equal(together[i, r], want[i, t])
    assert together.any(-1).sum() == n * T and all(k.view(R, rb + 16).any(-1).sum() == T for k in apart)
    with pytest.raises(avsg.AvsgError):                                                # memory that the GPU cannot reach
        avsg.append(latent, part, positions, [torch.zeros(R * rb + 16, dtype=torch.uint8).data_ptr() + 15 & ~15] * n, row_format=fmt)


def test_append_far_into_a_large_cache(avsg):
    import torch
    import rows_reference as ref
    R = 4_000_000
    kv = torch.empty(2, R, 1152, dtype=torch.uint8, device="cuda")
    kv[:, -2:] = 0
    x, part = torch.randn(2, 1, 512, device="cuda").to(torch.bfloat16), torch.randn(2, 1, 64, device="cuda").to(torch.bfloat16)
    avsg.append(x, part, torch.full((2, 1), R - 1, dtype=torch.int32, device="cuda"), kv, row_format=0)
    assert torch.equal(kv[:, -1], torch.cat((x, part), 2)[:, 0].contiguous().view(torch.uint8)) and not kv[:, -2].any()


def test_append_captured_with_attention(avsg):
    # a decode step's append and its attention in one graph: positions move between replays
    import torch
    import rows_reference as ref
    n, T, H, S = 2, 1, 16, 64
    g = _gen(34)
    latent = torch.zeros(n, T, 512, dtype=torch.bfloat16, device="cuda")
    part = torch.zeros(n, T, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(n, T, H, 576, dtype=torch.bfloat16, device="cuda")
    positions = torch.zeros(n, T, dtype=torch.int32, device="cuda")
    cache = torch.zeros(n, S, 656, dtype=torch.uint8, device="cuda")
    slots = torch.full((n, T, S), -1, dtype=torch.int32, device="cuda")
    rope = avsg.Rope(INV_FREQ)

    def step():
        avsg.append(latent, part, positions, cache, row_format=1, rope=rope)
        return avsg.attend(q, cache, slots, row_format=1, scale=SCALE, want_lse=True, rope=rope, positions=positions)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for t in range(5):
        latent.copy_(torch.randn(n, T, 512, generator=g, device="cuda"))
        part.copy_(torch.randn(n, T, 64, generator=g, device="cuda"))
        q.copy_(torch.randn(n, T, H, 576, generator=g, device="cuda"))
        positions.fill_(t)
        slots[:, :, t] = t
        graph.replay()
        ref.agree(*got, ref.attend(q, cache, slots, 1, SCALE, positions=positions, inv_freq=INV_FREQ))
    turned = ref.turn(part, positions, INV_FREQ)
    _rows_agree(cache[:, 4], ref.pack(latent.double().view(-1, 512), turned.to(torch.bfloat16).view(-1, 64), 1), 1, turned[:, 0])


# ---- the path as a serving program runs it -----------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
def test_append_step_attend(avsg, fmt):
    """Rows appended to pinned memory, fetched into slots by avsg_step, read by avsg_attend through its slot table; predicted tokens
    that were not accepted are appended again with other contents."""
    import torch
    import rows_reference as ref
    n, T, K, S, H, context = 3, 2, 48, 128, 12, 400
    g = _gen(35)
    rb = ref.BYTES[fmt]
    rope = avsg.Rope(INV_FREQ)
    ctx = avsg.Context(num_tables=n, buffer_slots=S, row_bytes=rb, max_topk=K, max_tokens=T)
    kv = [avsg.pinned_empty(context * rb) for _ in range(n)]
    tables = [2, 0, 1]
    shadow = torch.zeros(n, context, rb, dtype=torch.uint8, device="cuda")

    def put(positions):
        t = positions.shape[1]
        latent = torch.randn(n, t, 512, generator=g, device="cuda").to(torch.bfloat16)
        part = torch.randn(n, t, 64, generator=g, device="cuda").to(torch.bfloat16)
        ctx.append(tables, latent, part, positions, kv, row_format=fmt, rope=rope, kv_rows=[context] * n)
        avsg.append(latent, part, positions, shadow, row_format=fmt, rope=rope)

    put(torch.arange(300, device="cuda", dtype=torch.int32).expand(n, 300).contiguous())          # the prompts
    at = 300
    for step in range(12):
        positions = torch.tensor([[at, at + 1]] * n, dtype=torch.int32, device="cuda")
        put(positions)
        accepted = at + 1 + step % 2
        ids = torch.stack([torch.stack([torch.cat((torch.randperm(at - 1, generator=g, device="cuda")[:K - 2 - t], positions[i, :1 + t],
                                                   torch.full((1,), -1, device="cuda")))
                                        for t in range(T)]) for i in range(n)]).to(torch.int32)
        out = ctx.step(tables, ids, kv, [accepted] * n, kv_rows=[context] * n)
        q = torch.randn(n, T, H, 576, generator=g, device="cuda").to(torch.bfloat16)
        got = ctx.attend(tables, q, out.slots, row_format=fmt, scale=SCALE, want_lse=True, rope=rope, positions=positions)
        want = ref.attend(q, shadow, ids, fmt, SCALE, positions=positions, inv_freq=INV_FREQ)
        ref.agree(*got, want)
        at = accepted
    assert ctx.sync_status() == 0
    beyond = torch.full((n, 1), context, dtype=torch.int32, device="cuda")
    ctx.append(tables, torch.zeros(n, 1, 512, device="cuda"), torch.zeros(n, 1, 64, device="cuda"), beyond, kv, row_format=fmt, kv_rows=[context] * n)
    assert ctx.sync_status() == avsg.STATUS_BAD_ID
    ctx.clear_status()
    with pytest.raises(avsg.AvsgError):
        ctx.append([0, 0, 1], torch.zeros(n, 1, 512, device="cuda"), torch.zeros(n, 1, 64, device="cuda"), beyond, kv, row_format=fmt)
    with pytest.raises(avsg.AvsgError):
        ctx.append(tables, torch.zeros(n, 1, 512, device="cuda"), torch.zeros(n, 1, 64, device="cuda"), beyond, kv, row_format=(fmt + 1) % 3)
