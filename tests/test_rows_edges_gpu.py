"""avsg_append and avsg_attend at the calls that their documentation allows and that are easy to get wrong: buffers and streams in
unusual places, caps far above the scores, groups of tiny numbers, outputs that hold something else before."""
import pytest

from test_rows_calls_gpu import _both, binding                                   # noqa: F401 (a fixture)
from test_rows_gpu import FORMATS, INV_FREQ, SCALE, _gen, _problem, avsg          # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def _ways(binding, call):                                                        # noqa: F811
    """What `call` returns with the extension module and without it; both are held until both are there."""
    b, module = binding
    got = []
    for way in (module, False):
        b._tensor_calls = way
        got.append(call())
    b._tensor_calls = module
    return got


def _refused(avsg, binding, call):                                               # noqa: F811
    x, y = _both(binding, call)
    for e in (x, y):
        assert isinstance(e, avsg.AvsgError) and e.code == avsg.EINVAL, e
    assert str(x) == str(y)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_buffer_whose_rows_share_their_place_is_refused(avsg, binding, fmt):    # noqa: F811
    # (a row that is expanded has strides of 0, which the C entry takes for the bytes of a row)
    q, buffer, slots = _problem(fmt, 2, 1, 4, 8, 32, seed=81)
    size = buffer.shape[2]
    for held in (buffer[:1, :1].expand(2, 32, size), buffer[:, :1].expand(2, 32, size), buffer[:1].expand(2, 32, size),
                 buffer.as_strided((2, 32, size), (32 * 16, 16, 1)), buffer.as_strided((2, 1, size), (0, 0, 1))):
        _refused(avsg, binding, lambda: avsg.attend(q, held, slots * 0, row_format=fmt, scale=SCALE))
    _refused(avsg, binding, lambda: avsg.attend(q[:1], buffer[:1, :1].expand(1, 32, size), slots[:1], row_format=fmt, scale=SCALE))


@pytest.mark.parametrize("fmt", FORMATS)
def test_tables_of_one_row_with_room_behind_them(avsg, binding, fmt):             # noqa: F811
    # one slot per table: the tables are apart by the first stride, whatever the second (of a single row) says
    import torch
    import rows_reference as ref
    n, T, H = 3, 2, 8
    q, buffer, slots = _problem(fmt, n, T, H, 1, 1, seed=80)
    want = ref.attend(q, buffer, slots, fmt, SCALE)
    size = buffer.shape[2]
    roomy = torch.full((n, 1, size + 48), 255, dtype=torch.uint8, device="cuda")
    roomy[..., :size] = buffer
    wide = torch.full((n, 5, size), 255, dtype=torch.uint8, device="cuda")
    wide[:, 3] = buffer[:, 0]
    for held in (roomy[..., :size], wide[:, 3:4], buffer, buffer.as_strided((n, 1, size), (size, 16, 1))):
        for got in _ways(binding, lambda: avsg.attend(q, held, slots, row_format=fmt, scale=SCALE, want_lse=True)):
            ref.agree(*got, want)


def _held_by_the_current_stream(like):
    """A tensor of that shape and type, dropped while a copy of it is still to be made on the current stream; the copy, what it
    has to hold, and the place of the dropped one."""
    import torch
    x = torch.empty_like(like)
    x.fill_(3.0)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                       # about 0.1 s
    return x.clone(), x.data_ptr()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("handle", [False, True], ids=["stream", "handle"])
def test_outputs_of_a_call_on_another_stream(avsg, binding, fmt, handle):         # noqa: F811
    # A block that was freed on the current stream may still be read by what is queued there: a call on another stream must not
    # be given it.  And a result that is dropped while the current stream still has to read it is not written by the next call.
    import torch
    n, T, H, K, S = 16, 2, 128, 64, 128
    q, buffer, slots = _problem(fmt, n, T, H, K, S, seed=82)
    latent, part = q[..., 0, :512], q[..., 0, 512:]
    positions = torch.arange(T, dtype=torch.int32, device="cuda").expand(n, T).contiguous()
    many = torch.randn(4, 4096, 576, generator=_gen(83), device="cuda").to(torch.bfloat16)
    at = torch.arange(4096, dtype=torch.int32, device="cuda").expand(4, 4096).contiguous()
    cache = torch.zeros(4, 4096, buffer.shape[2], dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    on = side.cuda_stream if handle else side
    calls = [lambda s: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True, stream=s)[0],
             lambda s: avsg.append(many[..., :512], many[..., 512:], at, cache, row_format=fmt, want_values=True, stream=s)]
    b, module = binding
    for call in calls:
        want = call(None).clone()
        for way in (module, False):
            b._tensor_calls = way
            torch.cuda.synchronize()
            torch.cuda.empty_cache()
            kept, place = _held_by_the_current_stream(want)
            out = call(on)
            assert out.data_ptr() != place
            side.synchronize()
            torch.cuda.synchronize()
            assert bool((kept == 3.0).all()), "a block that queued work still reads was written"
            assert torch.equal(out, want)
            # the result, read late by the current stream and dropped at once
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda._sleep(200_000_000)
            late = out.clone()
            place = out.data_ptr()
            del out
            again = torch.empty_like(want).fill_(0)      # (of the current stream: may not be that block either)
            out = call(on)
            assert out.data_ptr() != place
            with torch.cuda.stream(side):
                out.fill_(5.0)
            torch.cuda.synchronize()
            assert torch.equal(late, want), "a result that queued work still reads was written"
            del again
        b._tensor_calls = module


def test_a_call_on_the_default_stream_by_its_handle(avsg, binding):               # noqa: F811
    # 0 and 1 (the legacy stream's own handle) name the default stream, also while another one is current
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(1, 2, 1, 16, 64, 128, seed=84)
    want = ref.attend(q, buffer, slots, 1, SCALE)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = [x for s in (0, 1) for x in _ways(binding, lambda: avsg.attend(q, buffer, slots, row_format=1, scale=SCALE, want_lse=True, stream=s))]
    torch.cuda.synchronize()
    for x in got:
        ref.agree(*x, want)


def test_outputs_of_a_captured_call_on_another_stream(avsg, binding):             # noqa: F811
    # the call's stream joins a capture that another stream began
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(1, 2, 1, 16, 64, 128, seed=85)
    want = ref.attend(q, buffer, slots, 1, SCALE)
    side = torch.cuda.Stream()
    b, module = binding
    for way in (module, False):
        b._tensor_calls = way
        avsg.attend(q, buffer, slots, row_format=1, scale=SCALE)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            side.wait_stream(torch.cuda.current_stream())
            got = avsg.attend(q, buffer, slots, row_format=1, scale=SCALE, want_lse=True, stream=side)
            torch.cuda.current_stream().wait_stream(side)
        got[0].zero_()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        ref.agree(*got, want)
    b._tensor_calls = module


def test_outputs_of_a_step_on_another_stream(avsg):                               # noqa: F811
    # as above, for the slot table of Context.step
    import torch
    n, T, K, N = 4, 1, 2048, 4096
    ctx = avsg.Context(num_tables=n, buffer_slots=4096, row_bytes=400, max_topk=K, max_tokens=T)
    try:
        kv = [torch.zeros(N, 400, dtype=torch.uint8, device="cuda") for _ in range(n)]
        ids = torch.stack([torch.randperm(N, generator=_gen(86), device="cuda")[:K] for _ in range(n * T)]).to(torch.int32).view(n, T, K)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        kept, place = _held_by_the_current_stream(ids)
        out = ctx.step([0, 1, 2, 3], ids, kv, [N] * n, stream=side)
        assert place not in (out.slots.data_ptr(), out.hit.data_ptr(), out.miss_count.data_ptr())
        torch.cuda.synchronize()
        assert bool((kept == 3).all())
        again = ctx.step([0, 1, 2, 3], ids, kv, [N] * n)
        torch.cuda.synchronize()
        assert torch.equal(out.slots, again.slots) and ctx.sync_status() == 0
    finally:
        ctx.close()


CAPS = [2.0 ** -126, 1e-30, 0.5, 3.0, 15.0, 50.0, 1e3, 1e5, 1e7, 1e10, 2.0 ** 100, 2.0 ** 126, 3.4028234e38]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", [1e-3, 1.0, 300.0])
def test_capped_scores_keep_their_digits_under_any_cap(avsg, fmt, size):          # noqa: F811
    """One row to a query: lse is its score.  The same call without a cap gives the score z that goes into the cap.

    The bound.  |z| / cap < 0.6: tanh(y) / y as a polynomial, off by 2^-23 of itself, two more roundings.  Else 1 - 2 / (1 + exp2(.)): the
    argument is off by 5 x 2^-24 of itself (scale, cap and constant rounded, two products), which moves tanh by y sech(y)^2 of that, 2.1 x
    2^-24 at most; exp2 is off by 2^-22.5, of which sech(y)^2 / 2 <= 0.36 arrives; the quotient by 2^-22 of its 0.47 or less, the two sums by
    2^-24 of 0.5 and 1: 6 x 2^-24 together where tanh is 0.54 or more, and three roundings of the product: 14 x 2^-24.  2^-20 covers both;
    the two logarithms' own rounding is 4 x 2^-24.  Results below 2^-126 may count as zero."""
    import torch
    q, buffer, slots = _problem(fmt, 4, 4, 64, 1, 64, seed=87)
    scale = SCALE * size
    _, plain = avsg.attend(q, buffer, slots, row_format=fmt, scale=scale, want_lse=True)
    z = plain.double()
    assert z.abs().max() > size and (z.abs() < size).any()
    for cap in CAPS:
        out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=scale, want_lse=True, softcap=cap)
        want = cap * torch.tanh(z / cap)
        off = (lse.double() - want).abs()
        allowed = want.abs() * (2.0 ** -20 + 2.0 ** -22) + 2.0 ** -124
        assert bool((off <= allowed).all()), "cap %g: off by %.3g of %.3g allowed" % (cap, *(x[(off - allowed).argmax()].item() for x in (off.flatten(), allowed.flatten())))
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("cap", [1e5, 1e8, 3.4028234e38])
def test_attention_under_a_cap_far_above_its_scores(avsg, fmt, cap):              # noqa: F811
    # cap x tanh(z / cap) is z to within z (z / cap)^2, far below a rounding: the bounds are those without a cap
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 2, 2, 24, 300, 512, seed=88)
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True, softcap=cap)
    _, _, eo, el = ref.attend(q, buffer, slots, fmt, SCALE)
    want, want_lse, _, _ = ref.attend(q, buffer, slots, fmt, SCALE, softcap=cap)
    ref.agree(out, lse, (want, want_lse, eo, el))


@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_append_of_tiny_groups(avsg, fmt, dtype):                                 # noqa: F811
    # groups down to where magnitudes count as zero (2^-126): codes are still the nearest to number / scale itself
    import torch
    import rows_reference as ref
    T = 400
    g = _gen(89)
    size = torch.exp2(-90.0 - 36.0 * torch.arange(T, device="cuda", dtype=torch.float64) / T)[:, None]
    x = torch.randn(T, 512, generator=g, device="cuda", dtype=torch.float64) * size
    x[::2, 1::2] = torch.round(x[::2, 1::2] / size[::2] * 16) / 16 * size[::2]     # (few bits: next to ties, or on them)
    x = x.to(getattr(torch, dtype))
    x = torch.where(x.double().abs() < 2.0 ** -126, torch.zeros_like(x), x)[None]
    part = torch.zeros(1, T, 64, device="cuda", dtype=x.dtype)
    positions = torch.arange(T, device="cuda", dtype=torch.int32)[None]
    kv = torch.zeros(1, T, ref.BYTES[fmt], dtype=torch.uint8, device="cuda")
    avsg.append(x, part, positions, kv, row_format=fmt)
    want = ref.pack(x[0].double(), part[0].to(torch.bfloat16), fmt)
    assert torch.equal(kv[0], want), "%d bytes differ" % int((kv[0] != want).sum())


@pytest.mark.parametrize("fmt", [1, 2])
def test_values_of_tiny_groups(avsg, fmt):                                        # noqa: F811
    # what the rows stand for, down to 2^-126; the smallest scale of 4-bit rows, 2^-127, is below that itself
    import torch
    import rows_reference as ref
    T = 64
    x = torch.randn(T, 512, generator=_gen(93), device="cuda") * torch.exp2(-118.0 - 9.0 * torch.arange(T, device="cuda") / T)[:, None]
    x = torch.where(x.abs() < 2.0 ** -126, torch.zeros_like(x), x)[None]
    part = torch.zeros(1, T, 64, device="cuda")
    positions = torch.arange(T, device="cuda", dtype=torch.int32)[None]
    kv = torch.zeros(1, T, ref.BYTES[fmt], dtype=torch.uint8, device="cuda")
    values = avsg.append(x, part, positions, kv, row_format=fmt, want_values=True)[0].double()
    assert torch.equal(kv[0], ref.pack(x[0].double(), part[0].to(torch.bfloat16), fmt))
    stands = ref.unpack(kv[0], fmt).float().to(torch.bfloat16).double()
    small = stands.abs() < 2.0 ** -126
    assert torch.equal(values[~small], stands[~small]) and bool((values[small].abs() < 2.0 ** -126).all()) and bool(small.any()) and bool((~small).any())


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_status_word_elsewhere_is_refused(avsg, binding, fmt):                  # noqa: F811
    # (the calls have nothing to report)
    import torch
    q, buffer, slots = _problem(fmt, 2, 1, 4, 8, 32, seed=90)
    positions = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    for status in (torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32).pin_memory()):
        _refused(avsg, binding, lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, status=status))
        _refused(avsg, binding, lambda: avsg.append(q[..., 0, :512], q[..., 0, 512:], positions, buffer, row_format=fmt, status=status))


@pytest.mark.parametrize("fmt", FORMATS)
def test_more_rows_than_a_cache_tensor_has_are_refused(avsg, binding, fmt):       # noqa: F811
    # (the calls' positions lie within the tensors)
    import torch
    bytes_ = avsg.row_bytes(fmt)
    n, R = 2, 6
    latent, part = torch.ones(n, 1, 512, device="cuda"), torch.ones(n, 1, 64, device="cuda")
    positions = torch.tensor([[5], [0]], dtype=torch.int32, device="cuda")
    pool = torch.zeros(n, R, bytes_, dtype=torch.uint8, device="cuda")
    apart = [torch.zeros(R * bytes_, dtype=torch.uint8, device="cuda") for _ in range(n)]
    pinned = [avsg.pinned_empty(R * bytes_) for _ in range(n)]
    huge = [avsg.pinned_empty(R * bytes_, huge_pages=True) for _ in range(n)]
    for kv in (pool, pool[0], apart, pinned, huge, [apart[0].data_ptr(), pinned[0]]):
        for rows in ([R, R + 1], [R], [R] * 3):
            _refused(avsg, binding, lambda: avsg.append(latent, part, positions, kv, row_format=fmt, kv_rows=rows))
        for got in _both(binding, lambda: avsg.append(latent, part, positions, kv, row_format=fmt, kv_rows=[R, R])):
            assert got is None
    # without kv_rows: what a table's own cache has no room for is reported, whatever the others are given as
    late = torch.tensor([[5], [R]], dtype=torch.int32, device="cuda")
    for kv in (pinned, huge, [apart[0].data_ptr(), apart[1]]):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        avsg.append(latent, part, late, kv, row_format=fmt, status=status)
        assert int(status) == avsg.STATUS_BAD_ID
    wide = [torch.zeros(R, bytes_ + 16, dtype=torch.uint8, device="cuda") for _ in range(n)]
    _refused(avsg, binding, lambda: avsg.append(latent, part, positions, wide, row_format=fmt, row_stride=[bytes_ + 16] * n, kv_rows=[R + 1, R]))
    _refused(avsg, binding, lambda: avsg.append(latent, part, positions, apart, row_format=fmt, row_stride=[bytes_]))
    # addresses have no limit of their own
    for got in _both(binding, lambda: avsg.append(latent, part, positions, [k.data_ptr() for k in apart], row_format=fmt, kv_rows=[R] * n)):
        assert got is None
    torch.cuda.synchronize()
    assert all(k.view(R, bytes_)[p].any() for k, p in zip(apart, (5, 0)))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", [2.0 ** 40, 2.0 ** 95])
def test_large_values_under_scores_that_rise(avsg, fmt, size):                    # noqa: F811
    # Scores (of the rotated part alone) rise by 2^55 along the list, so that weights are taken against maxima of the past; what is
    # summed up meanwhile must not leave the range of 32 bits.
    import torch
    import rows_reference as ref
    K, H = 2048, 4
    g = _gen(94)
    x = torch.randn(K, 512, generator=g, device="cuda", dtype=torch.float64) * size
    r = torch.zeros(K, 64, device="cuda", dtype=torch.bfloat16)
    r[:, 0] = torch.arange(K, device="cuda") // 64 * 64.0
    r[:, 1] = torch.arange(K, device="cuda") % 64
    buffer = ref.pack(x, r, fmt)[None].contiguous()
    q = torch.zeros(1, 1, H, 576, device="cuda", dtype=torch.bfloat16)
    q[..., 512] = q[..., 513] = torch.tensor([1.0, 0.5, -1.0, 0.0], device="cuda", dtype=torch.bfloat16)
    slots = torch.arange(K, device="cuda", dtype=torch.int32).view(1, 1, K)
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=38.0 / K, want_lse=True)
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, 38.0 / K))


@pytest.mark.parametrize("fmt", FORMATS)
def test_numbers_and_status_words_that_do_not_fit_are_refused(avsg, binding, fmt):               # noqa: F811
    import torch
    q, buffer, slots = _problem(fmt, 2, 1, 4, 8, 32, seed=95)
    latent, part, positions = q[..., 0, :512], q[..., 0, 512:], torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    for kw in (dict(scale=1e300), dict(scale=SCALE, softcap=1e39), dict(scale=SCALE, softcap=1 << 200)):
        _refused(avsg, binding, lambda: avsg.attend(q, buffer, slots, row_format=fmt, **kw))
    ctx = avsg.Context(num_tables=2, buffer_slots=32, row_bytes=avsg.row_bytes(fmt), max_topk=8)
    try:
        for wrong in (-1, 1 << 40):
            _refused(avsg, binding, lambda: ctx.attend([0, 1], q, slots, row_format=wrong, scale=SCALE))
            _refused(avsg, binding, lambda: avsg.append(latent, part, positions, [buffer[0], buffer[1]], row_format=wrong))
    finally:
        ctx.close()
    for status in (torch.zeros(4, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"),
                   torch.zeros(0, dtype=torch.int32, device="cuda")):
        _refused(avsg, binding, lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, status=status))
        _refused(avsg, binding, lambda: avsg.append(latent, part, positions, buffer, row_format=fmt, status=status))


@pytest.mark.parametrize("size", [2.0 ** 8, 2.0 ** 10, 2.0 ** 12])
@pytest.mark.parametrize("fmt", FORMATS)
def test_queries_with_a_few_large_numbers(avsg, fmt, size):                       # noqa: F811
    # Numbers below 2^-9 of a head's largest are rounded to 2^-17 of it with 8-bit rows, and with them only (the reference's bound has
    # that term for this format alone).  Keys are small where the queries are large, so that it is the small numbers that decide.
    import torch
    import rows_reference as ref
    q, buffer, slots = _problem(fmt, 2, 2, 20, 200, 256, seed=91)
    x = ref.unpack(buffer.view(-1, buffer.shape[2]), fmt)
    large = [3, 140, 300]
    x[:, large] /= size
    buffer = ref.pack(x[:, :512], x[:, 512:].to(torch.bfloat16), fmt).view(buffer.shape)
    q[..., large] = (q[..., large].float() * size).to(torch.bfloat16)
    out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True)
    ref.agree(out, lse, ref.attend(q, buffer, slots, fmt, SCALE))


@pytest.mark.parametrize("fmt", FORMATS)
def test_outputs_are_written_whole_and_nothing_beside_them(avsg, binding, fmt):   # noqa: F811
    # the caller's outputs hold something else before each way; what a call allocates is kept while the other way runs
    import torch
    import rows_reference as ref
    n, T, H, K = 2, 3, 20, 70
    q, buffer, slots = _problem(fmt, n, T, H, K, 128, seed=92)
    slots[1, 2] = -1
    want = ref.attend(q, buffer, slots, fmt, SCALE)
    b, module = binding
    wide = torch.empty(n, T, H, 528, dtype=torch.bfloat16, device="cuda")
    lses = torch.empty(3, n, T, H, device="cuda")
    for way in (module, False):
        b._tensor_calls = way
        wide.fill_(float("nan"))
        lses.fill_(float("nan"))
        out, lse = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, out=wide[..., 8:520], lse=lses[1])
        ref.agree(out, lse, want)
        assert wide[..., :8].isnan().all() and wide[..., 520:].isnan().all() and lses[::2].isnan().all()
    b._tensor_calls = module
    for got in _ways(binding, lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True)):
        ref.agree(*got, want)
    latent, part = q[:, :, 0, :512], q[:, :, 0, 512:]
    positions = torch.tensor([[0, 1, 2], [4, -1, 3]], dtype=torch.int32, device="cuda")
    written = positions >= 0
    stands = ref.unpack(ref.pack(latent.double().reshape(-1, 512), part.reshape(-1, 64), fmt), fmt).view(n, T, 576).float().to(torch.bfloat16)
    values = torch.empty(3, n, T, 576, dtype=torch.bfloat16, device="cuda")
    for way in (module, False):
        b._tensor_calls = way
        values.fill_(float("nan"))
        kv = torch.full((n, 5, buffer.shape[2]), 17, dtype=torch.uint8, device="cuda")
        assert avsg.append(latent, part, positions, kv, row_format=fmt, values=values[1]) is not None
        assert torch.equal(values[1][written], stands[written]) and values[1][~written].isnan().all() and values[::2].isnan().all()
    b._tensor_calls = module
    for got in _ways(binding, lambda: avsg.append(latent, part, positions, kv, row_format=fmt, want_values=True)):
        assert torch.equal(got[written], stands[written])


def test_calls_of_a_closed_context_are_refused(avsg, binding):                   # noqa: F811
    import torch
    q, buffer, slots = _problem(1, 2, 1, 4, 8, 32, seed=96)
    ctx = avsg.Context(num_tables=2, buffer_slots=32, row_bytes=656, max_topk=8)
    ctx.close()
    positions = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    _refused(avsg, binding, lambda: ctx.attend([0, 1], q, slots, row_format=1, scale=SCALE))
    _refused(avsg, binding, lambda: ctx.append([0, 1], q[..., 0, :512], q[..., 0, 512:], positions, buffer, row_format=1))
