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
