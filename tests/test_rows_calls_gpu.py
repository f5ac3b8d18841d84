"""avsg_append and avsg_attend through both ways of the binding (the extension module, and marshalled in Python): the same
results, the same refusals."""
import pytest

from test_rows_gpu import FORMATS, INV_FREQ, SCALE, _gen, _problem, avsg      # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture
def binding(avsg):                                                            # noqa: F811
    from paper_2609_37538_b200 import binding as b
    b._rows_functions()
    assert b._tensor_calls, "the extension module is not built"
    module = b._tensor_calls
    yield b, module
    b._tensor_calls = module


def _both(binding, call):
    """What `call` answers with the module, and without it."""
    b, module = binding
    got = []
    for way in (module, False):
        b._tensor_calls = way
        try:
            got.append(call())
        except Exception as e:                                                # noqa: BLE001 (what is raised is compared)
            got.append(e)
    b._tensor_calls = module
    return got


def _same(x, y):
    import torch
    if isinstance(x, (tuple, list)):
        return type(x) is type(y) and len(x) == len(y) and all(_same(a, b) for a, b in zip(x, y))
    if torch.is_tensor(x):
        return torch.is_tensor(y) and x.dtype == y.dtype and x.shape == y.shape and torch.equal(x.float(), y.float())
    return x is y or x == y


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_both_ways(avsg, binding, fmt):                                # noqa: F811
    import torch
    b, module = binding
    n, T, H, K, S = 2, 2, 24, 100, 256
    q, buffer, slots = _problem(fmt, n, T, H, K, S, seed=1)
    rope = avsg.Rope(INV_FREQ)
    g = _gen(2)
    positions = torch.randint(0, 5000, (n, T), generator=g, device="cuda", dtype=torch.int32)
    ids = torch.randint(0, 5000, (n, T, K), generator=g, device="cuda", dtype=torch.int32)
    spans = torch.tensor([[100, 4000]], device="cuda", dtype=torch.int32).expand(n, T, 2).contiguous()
    slopes = torch.rand(H, generator=g, device="cuda") * 1e-3
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    wide = torch.empty(n, T, H, 520, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(n, T, H, device="cuda")
    some = [
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=1, want_lse=1),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, lse=lse, out=wide[..., :512]),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, want_lse=True, rope=rope, positions=positions, ids=ids, spans=spans,
                            slopes=slopes, softcap=20.0, status=status),
        lambda: avsg.attend(q[:1], buffer[:1, :100], slots[:1].clamp(max=99), row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, stream=side),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, stream=side.cuda_stream),
        lambda: avsg.attend(torch.nn.Parameter(q), buffer, slots, row_format=fmt, scale=SCALE),
    ]
    for call in some:
        torch.cuda.synchronize()
        got = []
        for way in (module, False):
            b._tensor_calls = way
            x = call()
            torch.cuda.synchronize()
            got.append([t.clone() for t in x] if isinstance(x, tuple) else x.clone())
        b._tensor_calls = module
        assert _same(*got)
    assert int(status) == 0
    out = avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, out=wide[..., :512])
    assert out.data_ptr() == wide.data_ptr()
    refused = [
        lambda: avsg.attend(q.half(), buffer, slots, row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q[..., :575], buffer, slots, row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q.transpose(2, 3), buffer, slots, row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q.cpu(), buffer, slots, row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q, buffer[:, :100], slots, row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q, buffer[:1], slots, row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q, buffer, slots.long(), row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q, buffer, slots[:, :, ::2], row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q, buffer, slots[:, :1], row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q, buffer, slots, row_format=3, scale=SCALE),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=float("nan")),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, softcap=-1.0),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, slopes=slopes),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, slopes=slopes[:-1], ids=ids, positions=positions),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, spans=spans),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, rope=rope),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, out=wide),
        lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, lse=lse.half()),
        lambda: avsg.attend(q[:0], buffer[:0], slots[:0], row_format=fmt, scale=SCALE),
        lambda: avsg.attend(q[:, :, :0], buffer, slots, row_format=fmt, scale=SCALE),
    ]
    for k, call in enumerate(refused):
        x, y = _both(binding, call)
        assert type(x) is type(y) and isinstance(x, Exception) and str(x) == str(y), (k, x, y)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("type_", ["bfloat16", "float16", "float32"])
def test_append_both_ways(avsg, binding, fmt, type_):                         # noqa: F811
    import torch
    b, module = binding
    n, T, R = 3, 4, 16
    bytes_ = avsg.row_bytes(fmt)
    g = _gen(3)
    both = torch.randn(n, T, 576, generator=g, device="cuda").to(getattr(torch, type_))
    latent, part = both[..., :512], both[..., 512:]
    positions = torch.arange(T, device="cuda", dtype=torch.int32).expand(n, T).contiguous()
    rows = positions.flip(1).contiguous()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rope = avsg.Rope(INV_FREQ, halves=True)
    held = torch.zeros(n, R, bytes_ + 16, dtype=torch.uint8, device="cuda")
    shared = (positions + torch.arange(n, device="cuda", dtype=torch.int32)[:, None] * T).contiguous()
    given = torch.empty(n, T, 576, dtype=torch.bfloat16, device="cuda")
    some = [
        lambda kv: avsg.append(latent, part, positions, kv[..., :bytes_].contiguous().copy_(kv[..., :bytes_]), row_format=fmt),
        lambda kv: avsg.append(latent, part, positions, kv[..., :bytes_], row_format=fmt, rope=rope, want_values=1),
        lambda kv: avsg.append(latent, part, positions, kv[..., :bytes_], row_format=fmt, rope=rope, rows=rows, values=given, status=status),
        lambda kv: avsg.append(latent, part, shared, kv[0, :, :bytes_], row_format=fmt, rows=shared, want_values=True),
        lambda kv: avsg.append(latent[:1], part[:1], positions[:1], kv[:1, :, :bytes_], row_format=fmt),
        lambda kv: avsg.append(latent, part, positions, [k[:, :bytes_] for k in kv], row_format=fmt, row_stride=[bytes_ + 16] * n, kv_rows=[R] * n),
        lambda kv: avsg.append(latent, part, positions, kv[..., :bytes_], row_format=fmt, kv_rows=[R] * n),
    ]
    for call in some:
        got = []
        for way in (module, False):
            b._tensor_calls = way
            held.zero_()
            v = call(held)
            torch.cuda.synchronize()
            got.append((held.clone(), None if v is None else v.clone()))
        b._tensor_calls = module
        assert _same(*got)
    assert int(status) == 0
    kv = held[..., :bytes_]
    refused = [
        lambda: avsg.append(latent.double(), part.double(), positions, kv, row_format=fmt),
        lambda: avsg.append(latent, part.double(), positions, kv, row_format=fmt),
        lambda: avsg.append(latent[..., :511], part, positions, kv, row_format=fmt),
        lambda: avsg.append(latent, part[:, :2], positions, kv, row_format=fmt),
        lambda: avsg.append(latent, part, positions.long(), kv, row_format=fmt),
        lambda: avsg.append(latent, part, positions[:, :2], kv, row_format=fmt),
        lambda: avsg.append(latent, part, positions, kv[..., :-16], row_format=fmt),
        lambda: avsg.append(latent, part, positions, kv[:2], row_format=fmt),
        lambda: avsg.append(latent, part, positions, kv, row_format=7),
        lambda: avsg.append(latent, part, positions, kv, row_format=fmt, values=given.float()),
        lambda: avsg.append(latent[:0], part[:0], positions[:0], kv[:0], row_format=fmt),
    ]
    for k, call in enumerate(refused):
        x, y = _both(binding, call)
        assert type(x) is type(y) and isinstance(x, Exception) and str(x) == str(y), (k, x, y)


def test_calls_of_a_context_both_ways(avsg, binding):                         # noqa: F811
    import torch
    b, module = binding
    n, T, K, N = 2, 2, 64, 256
    fmt = avsg.ROW_FP8
    bytes_ = avsg.row_bytes(fmt)
    g = _gen(4)
    q = torch.randn(n, T, 20, 576, generator=g, device="cuda").to(torch.bfloat16)
    latent = torch.randn(n, N, 512, generator=g, device="cuda").to(torch.bfloat16)
    part = torch.randn(n, N, 64, generator=g, device="cuda").to(torch.bfloat16)
    positions = torch.arange(N, device="cuda", dtype=torch.int32).expand(n, N).contiguous()
    ids = torch.stack([torch.randperm(N, generator=g, device="cuda")[:K] for _ in range(n * T)]).to(torch.int32).view(n, T, K)
    got = []
    for way in (module, False):
        b._tensor_calls = way
        kv = torch.zeros(n, N, bytes_, dtype=torch.uint8, device="cuda")
        ctx = avsg.Context(num_tables=4, buffer_slots=512, row_bytes=bytes_, max_topk=K, max_tokens=T)
        try:
            ctx.append([2, 1], latent, part, positions, kv, row_format=fmt)
            step = ctx.step([2, 1], ids, [kv[0], kv[1]], [N, N])
            got.append(ctx.attend([2, 1], q, step.slots, row_format=fmt, scale=SCALE, want_lse=True) + (kv,))
            x = _both(binding, lambda: ctx.attend([2, 9], q, step.slots, row_format=fmt, scale=SCALE))
            assert all(isinstance(e, avsg.AvsgError) for e in x) and str(x[0]) == str(x[1])
            x = _both(binding, lambda: ctx.attend([2], q, step.slots, row_format=fmt, scale=SCALE))
            assert all(isinstance(e, avsg.AvsgError) for e in x) and str(x[0]) == str(x[1])
            x = _both(binding, lambda: ctx.append([2, 2], latent, part, positions, kv, row_format=fmt))
            assert all(isinstance(e, avsg.AvsgError) for e in x) and str(x[0]) == str(x[1])
            torch.cuda.synchronize()
        finally:
            ctx.close()
    assert _same(*got)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_to_a_list_of_tensors_stays_within_them(avsg, binding, fmt):   # noqa: F811
    import torch
    b, module = binding
    n, T, R = 2, 4, 6
    bytes_ = avsg.row_bytes(fmt)
    g = _gen(8)
    latent = torch.randn(n, T, 512, generator=g, device="cuda").to(torch.bfloat16)
    part = torch.randn(n, T, 64, generator=g, device="cuda").to(torch.bfloat16)
    positions = torch.tensor([[0, 5, 6, 7], [1, 2, 3, 9]], dtype=torch.int32, device="cuda")
    for way in (module, False):
        b._tensor_calls = way
        pool = torch.zeros(n, 12, bytes_, dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        avsg.append(latent, part, positions, [pool[0, :R], pool[1, :R]], row_format=fmt, status=status)
        assert int(status) == avsg.STATUS_BAD_ID
        written = (pool != 0).any(2).cpu()
        assert written[0].nonzero().flatten().tolist() == [0, 5] and written[1].nonzero().flatten().tolist() == [1, 2, 3]


@pytest.mark.parametrize("fmt", FORMATS)
def test_what_lies_elsewhere_or_shares_its_place_is_refused(avsg, binding, fmt):                   # noqa: F811
    import ctypes
    import torch
    b, module = binding
    q, buffer, slots = _problem(fmt, 2, 2, 8, 32, 64, seed=9)
    shared = torch.empty(1, 1, 1, 512, dtype=torch.bfloat16, device="cuda").expand(2, 2, 8, 512)
    for x in _both(binding, lambda: avsg.attend(q, buffer, slots, row_format=fmt, scale=SCALE, out=shared)):
        assert isinstance(x, avsg.AvsgError) and x.code == avsg.EINVAL
    # slots and positions in host memory, through the C entry with a context
    ctx = avsg.Context(num_tables=2, buffer_slots=64, row_bytes=avsg.row_bytes(fmt), max_topk=32, max_tokens=2)
    try:
        host = torch.zeros(2 * 2 * 32, dtype=torch.int32).pin_memory()
        out = torch.empty(2, 2, 8, 512, dtype=torch.bfloat16, device="cuda")
        ids = (ctypes.c_uint32 * 2)(0, 1)
        a = avsg.AvsgAttendArgs()
        a.n, a.n_tokens, a.topk, a.heads, a.row_format, a.scale = 2, 2, 32, 8, fmt, 1.0
        a.table_ids, a.slots, a.q, a.out = ctypes.addressof(ids), host.data_ptr(), q.data_ptr(), out.data_ptr()
        for k, (s, t) in enumerate(zip(q.stride(), out.stride())):
            if k < 3:
                a.q_stride[k], a.out_stride[k] = 2 * s, 2 * t
        assert avsg.load_library().avsg_attend(ctx._h, ctypes.byref(a), None) == avsg.EINVAL
        latent = torch.zeros(2, 2, 576, dtype=torch.bfloat16, device="cuda")
        kv = torch.zeros(2, 64, avsg.row_bytes(fmt), dtype=torch.uint8, device="cuda")
        p = avsg.AvsgAppendArgs()
        p.n, p.n_tokens, p.row_format, p.type = 2, 2, fmt, 0
        p.table_ids, p.latent, p.rope_part, p.positions, p.kv = ctypes.addressof(ids), latent.data_ptr(), latent.data_ptr() + 1024, host.data_ptr(), kv.data_ptr()
        for k in range(2):
            p.latent_stride[k] = p.rope_stride[k] = (2304, 1152)[k]
        p.kv_table_stride = 64 * avsg.row_bytes(fmt)
        assert avsg.load_library().avsg_append(ctx._h, ctypes.byref(p), None) == avsg.EINVAL
        torch.cuda.synchronize()
        assert ctx.sync_status() == 0
    finally:
        ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_queries_may_be_broadcast(avsg, binding, fmt):                        # noqa: F811
    import torch
    q, buffer, slots = _problem(fmt, 3, 2, 8, 40, 64, seed=10)
    one = q[:1, :1].expand(3, 2, 8, 576)
    for got in _both(binding, lambda: avsg.attend(one, buffer, slots, row_format=fmt, scale=SCALE)):
        assert torch.equal(got, avsg.attend(one.contiguous(), buffer, slots, row_format=fmt, scale=SCALE))
