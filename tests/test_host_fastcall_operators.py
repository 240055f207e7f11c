"""The binding's native marshaling of fs_rope, fs_rope_append and fs_batch_tables, on the CPU: its entry points are callbacks that
record what arrives; what it does not take, it answers None to."""
import ctypes

import pytest
import torch

import paper_2509_06261_amd as fs
from paper_2509_06261_amd import _fsfast, binding

vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
SIGNATURES = dict(rope=[vp, i32, vp, i64, i32, i32, vp, i64, i32, vp, i64, vp],
                  rope_append=[vp, i32, i32, vp, i64, i32, vp, i64, vp, i64, i32, vp, vp, vp, i32, i64, vp, vp],
                  batch_tables=[vp, i32, vp, vp, i32, vp, i64, vp, i32, vp, vp, vp, vp, vp, i64, vp, vp])
STREAM = 0x5EED0


@pytest.fixture(scope="module")
def got():
    seen = {}
    slow, binding._slow, binding._fast = binding._slow, lambda: None, binding._NotYet

    def recorder(name, types):
        def f(*args):
            seen[name] = list(args)
            return 7
        return ctypes.CFUNCTYPE(i32, *types)(f)

    seen["keep"] = [recorder(*x) for x in SIGNATURES.items()]
    address = [ctypes.cast(f, vp).value for f in seen["keep"]]
    _fsfast.init(torch.Tensor, torch.float16, torch.float32, torch.int32, ctypes.c_void_p, binding.fs_batch_t, binding.fs_append_t,
                 lambda: 3, lambda d: STREAM + d, *address[:1] * 5)
    x = torch.zeros((2, 1, 8), dtype=torch.float16)
    assert _fsfast.rope(vp(1), 0, x, torch.zeros(2, dtype=torch.int32), x, False, None) is None  # (not brought up yet)
    _fsfast.init_operators(torch.int64, *address)
    yield seen
    _fsfast.init()
    binding._slow = slow


def wide(n=5, heads=(6, 2, 2), d=16, dt=torch.float16):
    """Parts of one matrix."""
    x = torch.zeros((n, sum(heads) * d + 8), dtype=dt)
    return [p.view(n, -1, d) for p in x[:, :sum(heads) * d].split([h * d for h in heads], dim=1)], x.shape[1]


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("dt", [torch.float16, torch.float32])
def test_rope(got, dt):
    (x, _, _), step = wide(dt=dt)
    out, pos = torch.zeros((5, 6, 16), dtype=dt), ints(5)
    for inverse in (False, True):
        assert _fsfast.rope(vp(0x123), 2, x, pos, out, inverse, None) == 7
        src = fs.FS_SRC_FP32 if dt == torch.float32 else fs.FS_SRC_FP16
        assert got["rope"] == [0x123, 2, x.data_ptr(), step, 6, src, pos.data_ptr(), 5, int(inverse), out.data_ptr(), 96, STREAM + 3]
    one = x[:1]
    assert _fsfast.rope(vp(1), 2, one, ints(1), one, False, None) == 7 and got["rope"][3] == 96


@pytest.mark.parametrize("queries", [True, False])
def test_rope_append(got, queries):
    (q, k, v), step = wide()
    out, seq, pos, table = torch.zeros((5, 6, 16), dtype=torch.float16), ints(5), ints(5), ints(3, 4)
    a = [q if queries else None, k, v, seq, pos, table, out if queries else None]
    assert _fsfast.rope_append(vp(0x77), 1, 2, *a, None) == 7
    head = [q.data_ptr(), step, 6] if queries else [None, 0, 0]
    assert got["rope_append"] == [0x77, 1, 2, *head, k.data_ptr(), step, v.data_ptr(), step, fs.FS_SRC_FP16, seq.data_ptr(), pos.data_ptr(),
                                  table.data_ptr(), 4, 5, out.data_ptr() if queries else None, STREAM + 3]


@pytest.mark.parametrize("full", [True, False])
def test_batch_tables(got, full):
    held, new, ids, table, lens, off, seq, pos = ints(3), ints(3), ints(9), ints(3, 4), ints(3), ints(4), ints(20), ints(20)
    slots, status = torch.zeros(20, dtype=torch.int64), ints(1)
    a = [held if full else None, new, ids, table, lens, off, seq, pos, slots if full else None, status if full else None]
    assert _fsfast.batch_tables(vp(0x99), 1, *a, None) == 7
    p = [x.data_ptr() if x is not None else None for x in a]
    assert got["batch_tables"] == [0x99, 1, p[0], p[1], 3, p[2], 9, p[3], 4, *p[4:8], p[8], 20, p[9], STREAM + 3]


def test_the_unusual_is_left_to_ctypes(got):
    (q, k, v), _ = wide()
    out, seq, pos, table = torch.zeros((5, 6, 16), dtype=torch.float16), ints(5), ints(5), ints(3, 4)
    x = [q, k, v, seq, pos, table, out]
    for at, bad in ((0, q.float()), (0, q[:4]), (0, q.transpose(1, 2)), (0, None), (1, k.double()), (1, k[:, :1]), (2, v.float()), (2, v[..., ::2]), (3, ints(4)),
                    (3, seq.long()), (4, ints(10)[::2]), (5, table.T), (5, ints(4)), (6, out.float()), (6, None), (6, torch.zeros((5, 8, 16), dtype=torch.float16)[:, :6])):
        a = list(x)
        a[at] = bad
        assert _fsfast.rope_append(vp(1), 1, 2, *a, None) is None, (at, bad)
    assert _fsfast.rope_append(vp(1), 1, 2, *x, STREAM) is None
    assert _fsfast.rope_append(0x1234, 1, 2, *x, None) is None
    for a in ((k.transpose(0, 1), pos, out, False), (k, ints(4), k, False), (k, pos, v[:, :1], False), (k, pos, k.float(), False), (k, pos, k, 1), (k[0], pos, k[0], False)):
        assert _fsfast.rope(vp(1), 1, *a, None) is None
    good = [ints(3), ints(3), ints(9), table, ints(3), ints(4), ints(20), ints(20), torch.zeros(20, dtype=torch.int64), None]
    assert _fsfast.batch_tables(vp(1), 1, *good, None) == 7
    for at, bad in ((0, ints(2)), (1, ints(2)), (1, None), (2, ints(9).long()), (3, ints(12)), (3, ints(2, 4)), (3, table.T), (4, ints(4)), (5, ints(3)), (6, ints(19)),
                    (7, ints(40)[::2]), (8, ints(20)), (8, torch.zeros(19, dtype=torch.int64)), (9, 5)):
        a = list(good)
        a[at] = bad
        assert _fsfast.batch_tables(vp(1), 1, *a, None) is None, (at, bad)
    with pytest.raises(AssertionError):
        fs.fs_rope(vp(1), 1, k, ints(4), k)
    with pytest.raises(AssertionError):
        fs.fs_rope_append(vp(1), 1, 2, q, k, v.float(), seq, pos, table, out)
    with pytest.raises(AssertionError):
        fs.fs_batch_tables(vp(1), 1, *good[:4], ints(4), *good[5:])
