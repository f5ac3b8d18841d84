"""avsg_append and avsg_attend refuse what they do not serve, before anything touches a GPU."""
import ctypes

import pytest

import paper_2609_37538_b200 as avsg

P = 1 << 20          # an aligned address; refused calls never look behind it


def test_row_sizes():
    assert [avsg.row_bytes(f) for f in (avsg.ROW_BF16, avsg.ROW_FP8, avsg.ROW_FP4)] == [1152, 656, 400]
    assert avsg.load_library().avsg_row_bytes(3) == 0
    with pytest.raises(avsg.AvsgError):
        avsg.row_bytes(7)


def test_struct_layouts():
    assert ctypes.sizeof(avsg.AvsgRope) == 264
    assert ctypes.sizeof(avsg.AvsgAppendArgs) == 152
    assert ctypes.sizeof(avsg.AvsgAttendArgs) == 184


def test_rope_takes_32_frequencies():
    with pytest.raises(avsg.AvsgError):
        avsg.Rope([1.0] * 31)


def _append(**kw):
    a = avsg.AvsgAppendArgs()
    a.n, a.n_tokens, a.row_format, a.type = 1, 1, avsg.ROW_FP8, 0
    a.latent = a.rope_part = a.positions = a.kv = P
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(a, k)[v[0]] = v[1]
        else:
            setattr(a, k, v)
    return avsg.load_library().avsg_append(None, ctypes.byref(a), None)


def _array(kind, *values):
    a = (kind * len(values))(*values)
    _array.keep = getattr(_array, "keep", []) + [a]
    return ctypes.addressof(a)


@pytest.mark.parametrize("bad", [
    dict(n=0), dict(n=2049), dict(n_tokens=0), dict(n=2048, n_tokens=1 << 20), dict(row_format=3), dict(type=3), dict(latent=None),
    dict(rope_part=None), dict(positions=None), dict(kv=None), dict(latent=P + 8), dict(rope_part=P + 2), dict(kv=P + 8), dict(positions=P + 2),
    dict(rows=P + 1), dict(values=P + 4), dict(status=P + 2), dict(latent_stride=(1, 1000)), dict(rope_stride=(0, 8)), dict(kv_table_stride=24),
    dict(table_ids=P),
])
def test_append_refuses(bad):
    assert _append(**bad) == avsg.EINVAL


def test_append_refuses_bad_host_arrays():
    assert _append(kv_base=_array(ctypes.c_uint64, P)) == avsg.EINVAL                                   # kv and kv_base
    assert _append(kv=None, kv_base=_array(ctypes.c_uint64, 0)) == avsg.EINVAL
    assert _append(kv=None, kv_base=_array(ctypes.c_uint64, P + 4)) == avsg.EINVAL
    assert _append(row_stride=_array(ctypes.c_uint64, 640)) == avsg.EINVAL                              # shorter than a row
    assert _append(row_stride=_array(ctypes.c_uint64, 660)) == avsg.EINVAL
    assert _append(kv_rows=_array(ctypes.c_uint32, 0x80000001)) == avsg.EINVAL
    r = avsg.Rope([1.0] * 32)
    r.c.halves = 2
    assert _append(rope=ctypes.addressof(r.c)) == avsg.EINVAL
    r = avsg.Rope([1.0] * 31 + [float("inf")])
    assert _append(rope=ctypes.addressof(r.c)) == avsg.EINVAL
    assert avsg.load_library().avsg_append(None, None, None) == avsg.EINVAL


def _attend(**kw):
    a = avsg.AvsgAttendArgs()
    a.n, a.n_tokens, a.topk, a.heads, a.row_format, a.buffer_slots = 1, 1, 1, 1, avsg.ROW_FP8, 32
    a.slots = a.q = a.out = a.buffer = P
    a.scale = 1.0
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(a, k)[v[0]] = v[1]
        else:
            setattr(a, k, v)
    return avsg.load_library().avsg_attend(None, ctypes.byref(a), None)


@pytest.mark.parametrize("bad", [
    dict(n=0), dict(n=2049), dict(n_tokens=0), dict(topk=0), dict(heads=0), dict(row_format=3), dict(slots=None), dict(q=None), dict(out=None),
    dict(buffer=None), dict(buffer=P + 8), dict(q=P + 2), dict(out=P + 4), dict(slots=P + 2), dict(lse=P + 2), dict(status=P + 1),
    dict(q_stride=(2, 1000)), dict(out_stride=(0, 8)), dict(buffer_slots=0), dict(buffer_slots=0x80000001), dict(buffer_row_bytes=640),
    dict(buffer_row_bytes=664), dict(scale=float("nan")), dict(scale=float("inf")), dict(softcap=-1.0), dict(softcap=float("nan")),
    dict(spans=P), dict(slopes=P, ids=P), dict(slopes=P, positions=P), dict(table_ids=P), dict(ids=P + 2, spans=P), dict(spans=P + 2, ids=P),
])
def test_attend_refuses(bad):
    assert _attend(**bad) == avsg.EINVAL


def test_attend_refuses_sizes_and_rotation_without_positions():
    assert _attend(heads=1025) == avsg.EUNSUPPORTED
    assert _attend(n=2048, n_tokens=1 << 14) == avsg.EUNSUPPORTED
    assert _attend(topk=(1 << 24) + 1) == avsg.EUNSUPPORTED
    assert _attend(rope=ctypes.addressof(avsg.Rope([1.0] * 32).c)) == avsg.EINVAL
    assert avsg.load_library().avsg_attend(None, None, None) == avsg.EINVAL


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    import torch
    q = torch.zeros(1, 1, 1, 576, dtype=torch.bfloat16)
    with pytest.raises(avsg.AvsgError):
        avsg.attend(q, torch.zeros(1, 32, 656, dtype=torch.uint8), torch.zeros(1, 1, 1, dtype=torch.int32), row_format=avsg.ROW_FP8, scale=1.0)
    with pytest.raises(avsg.AvsgError):
        avsg.append(torch.zeros(1, 1, 512), torch.zeros(1, 1, 64), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, 4, 656, dtype=torch.uint8),
                    row_format=avsg.ROW_FP8)


@pytest.mark.parametrize("i,size", [(0, dict(n=2)), (1, dict(n_tokens=2)), (2, dict(heads=2))])
def test_attend_refuses_outputs_that_share_their_place(i, size):
    strides = [4096, 2048, 1024]
    strides[i] = 0
    a = avsg.AvsgAttendArgs()
    a.n = a.n_tokens = a.topk = a.heads = 1
    a.row_format, a.buffer_slots, a.scale = avsg.ROW_FP8, 32, 1.0
    a.slots = a.q = a.out = a.buffer = P
    for k, v in size.items():
        setattr(a, k, v)
    for k in range(3):
        a.out_stride[k] = strides[k]
    assert avsg.load_library().avsg_attend(None, ctypes.byref(a), None) == avsg.EINVAL


def test_rows_in_a_cache_given_as_a_tensor():
    import torch
    from paper_2609_37538_b200.binding import _rows_in
    flat = torch.zeros(10 * 656 + 100, dtype=torch.uint8)
    assert _rows_in(flat, 656, None) == 10 and _rows_in(flat[:655], 656, None) == 0 and _rows_in(flat[:0], 656, None) == 0
    assert _rows_in(flat[:6560].view(10, 656), 656, None) == 10
    wide = torch.zeros(7, 672, dtype=torch.uint8)
    assert _rows_in(wide[:, :656], 656, 672) == 7 and _rows_in(wide[:, :640], 656, 672) == 6
    assert _rows_in(torch.zeros(4, 164, dtype=torch.float32), 656, None) == 4


def test_attend_refuses_a_cap_that_counts_as_zero():
    assert _attend(softcap=1e-40) == avsg.EINVAL


def test_the_extension_module_serves_the_torch_that_it_was_built_for(monkeypatch):
    import torch
    from paper_2609_37538_b200 import binding as b
    b._rows_functions()
    module = b._tensor_calls
    try:
        if module:
            assert module.built_for == torch.__version__
        monkeypatch.setattr(torch, "__version__", "0.0.1")
        b._rows_functions()
        assert b._tensor_calls is False and b._attend_fn is not None
    finally:
        b._tensor_calls = module
