"""Host side of the FP8_BLOCK format, the rotary positions and the block tables (no GPU): geometry, frequencies, refusals; and the
plain implementations of tests/block_cache.py against hand-worked values."""
import numpy as np
import pytest

import block_cache as plain
import paper_2509_06261_amd as fs

FAKE_BASE = 0x7F0000000000
KiB = 1 << 10


@pytest.fixture()
def pool():
    p = fs.fs_pool_create(64 * KiB, 64 * 64 * KiB, FAKE_BASE)
    yield p
    fs.fs_pool_destroy(p)


@pytest.mark.parametrize("heads,d,layers,tokens", [(8, 128, 2, 63), (1, 8, 1, 1), (3, 64, 4, 31), (40, 128, 10, 7), (4, 256, 1, 16), (2, 512, 3, 5)])
def test_block_layout(heads, d, layers, tokens):
    want = plain.layout(heads, d, tokens, layers)
    assert fs.fs_block_bytes(fs.FS_KV_FP8_BLOCK, heads, d, layers, tokens) == want["block"]
    p = fs.fs_pool_create(want["block"], 4 * want["block"], FAKE_BASE)
    got, m = fs.fs_model_register_tokens(p, fs.FS_KV_FP8_BLOCK, heads, d, layers, tokens)
    g = fs.fs_model_geometry(p, m)
    assert got == g.tokens_per_block == tokens and g.kv_dtype == fs.FS_KV_FP8_BLOCK and g.param_bytes == 0
    assert (g.row_bytes, g.kv_tile, g.head_chunk, g.layer_bytes, g.block_bytes) == (d, want["tile"], want["chunk"], want["layer"], want["block"])
    assert heads * g.head_chunk + 8 * heads <= g.layer_bytes
    fs.fs_pool_destroy(p)


def test_tokens_per_block_leave_room_for_the_scales():
    for budget in (4 * KiB, 32 * KiB, 2048 * KiB):
        p = fs.fs_pool_create(budget, 8 * budget, FAKE_BASE)
        for heads, d, layers in ((1, 64, 1), (8, 128, 1), (2, 128, 2), (4, 64, 8)):
            fits = [t for t in range(1, budget // (2 * d * heads * layers) + 1) if plain.layout(heads, d, t, layers)["block"] <= budget]
            if fits:
                assert fs.fs_model_register(p, fs.FS_KV_FP8_BLOCK, heads, d, layers)[0] == max(fits)
            else:
                with pytest.raises(fs.FsError):
                    fs.fs_model_register(p, fs.FS_KV_FP8_BLOCK, heads, d, layers)
        fs.fs_pool_destroy(p)


SCALINGS = [("none", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)), ("wavelength", dict(factor=8.0, low=1.0, high=4.0, original=8192)),
            ("dimension", dict(factor=16.0, low=1.0, high=32.0, original=4096)), ("dimension", dict(factor=2.0, low=0.5, high=1e6, original=100))]
KINDS = dict(none=fs.FS_ROPE_UNSCALED, linear=fs.FS_ROPE_LINEAR, base=fs.FS_ROPE_BASE, wavelength=fs.FS_ROPE_WAVELENGTH, dimension=fs.FS_ROPE_DIMENSION)


@pytest.mark.parametrize("r", [4, 20, 64, 128, 512])
@pytest.mark.parametrize("scaling,par", SCALINGS)
def test_frequencies(r, scaling, par):
    for base in (10000.0, 500000.0):
        want = plain.frequencies(r, base, scaling, **par)
        kw = {"original_positions" if k == "original" else k: v for k, v in par.items()}
        got = fs.fs_rope_frequencies(fs.make_rope(r, base, scaling=KINDS[scaling], **kw))
        np.testing.assert_allclose(got, want, rtol=1e-13)


def test_frequencies_by_hand():
    f = fs.fs_rope_frequencies(fs.make_rope(4, 10000.0))
    np.testing.assert_allclose(f, [1.0, 0.01], rtol=1e-15)
    f = fs.fs_rope_frequencies(fs.make_rope(4, 10000.0, scaling=fs.FS_ROPE_BASE, factor=9.0))  # base * 9^2
    np.testing.assert_allclose(f, [1.0, 1 / 900.0], rtol=1e-15)
    # wavelengths 2 pi and 200 pi behind 100 pi original positions: 50 turns (kept), half a turn (stretched whole)
    f = fs.fs_rope_frequencies(fs.make_rope(4, 10000.0, scaling=fs.FS_ROPE_WAVELENGTH, factor=10.0, low=1.0, high=4.0, original_positions=314))
    np.testing.assert_allclose(f, [1.0, 0.001], rtol=1e-15)


GOOD = dict(rotary_dim=64, base=10000.0, scaling=fs.FS_ROPE_WAVELENGTH, factor=8.0, low=1.0, high=4.0, original_positions=8192)


@pytest.mark.parametrize("bad", [dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=-2), dict(rotary_dim=514), dict(base=1.0), dict(base=-5.0),
                                 dict(base=float("nan")), dict(base=float("inf")), dict(layout=2), dict(layout=-1), dict(scaling=5), dict(scaling=-1),
                                 dict(factor=0.0), dict(factor=float("nan")), dict(low=4.0), dict(low=-1.0), dict(high=float("inf")), dict(original_positions=0),
                                 dict(amplitude=0.0), dict(amplitude=float("nan")), dict(scaling=fs.FS_ROPE_DIMENSION, low=0.0),
                                 dict(scaling=fs.FS_ROPE_BASE, rotary_dim=2)])
def test_bad_rotations_are_refused(pool, bad):
    fs.fs_rope_frequencies(fs.make_rope(**GOOD))
    rope = fs.make_rope(**{**GOOD, **bad})
    for call in (lambda: fs.fs_rope_frequencies(rope), lambda: fs.fs_model_set_rope(pool, fs.fs_model_register(pool, fs.FS_KV_FP16, 2, 512, 1)[1], rope)):
        with pytest.raises(fs.FsError) as e:
            call()
        assert e.value.code == fs.FS_ERR_INVALID


def test_a_rotation_fits_its_model(pool):
    _, m = fs.fs_model_register(pool, fs.FS_KV_FP16, 2, 32, 1)
    for model, dim in ((m, 34), (m + 1, 32), (-1, 32)):
        with pytest.raises(fs.FsError) as e:
            fs.fs_model_set_rope(pool, model, fs.make_rope(dim, 10000.0))
        assert e.value.code == fs.FS_ERR_INVALID


A = FAKE_BASE  # a non-null, aligned address that a refused call never reads


def _append_args(**kw):
    a = dict(layer=0, q=A, q_stride=0, n_q=4, k=A, k_stride=0, v=A, v_stride=0, src=fs.FS_SRC_FP16, seq_idx=A, pos=A, tables=A, max_blocks=3, n=5, q_out=A)
    a.update(kw)
    return tuple(a.values())


@pytest.mark.parametrize("bad", [dict(layer=1), dict(layer=-1), dict(q=0), dict(q_out=0), dict(k=0), dict(v=0), dict(seq_idx=0), dict(pos=0), dict(tables=0),
                                 dict(max_blocks=0), dict(n=-1), dict(src=2), dict(n_q=-1), dict(q_stride=128), dict(k_stride=64), dict(v_stride=124),
                                 dict(q_stride=4 * 64 + 4), dict(q=A + 8), dict(k=A + 2), dict(v=A + 4), dict(q_out=A + 8), dict()])
def test_rope_append_refusals(pool, bad):
    """The last one has nothing wrong but that the model has no rotation."""
    L = fs.binding._L
    _, m = fs.fs_model_register(pool, fs.FS_KV_FP16, 2, 64, 1)
    assert L.fs_rope_append(pool, m, *_append_args(**bad), None) == fs.FS_ERR_INVALID
    assert fs.fs_last_error()
    assert L.fs_rope_append(pool, m + 1, *_append_args(), None) == fs.FS_ERR_INVALID
    assert L.fs_rope_append(None, m, *_append_args(), None) == fs.FS_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(x=0), dict(pos=0), dict(out=0), dict(heads=0), dict(n=-1), dict(src=7), dict(xs=64), dict(os=100), dict(x=A + 2), dict(out=A + 8), dict()])
def test_rope_refusals(pool, bad):
    L = fs.binding._L
    _, m = fs.fs_model_register(pool, fs.FS_KV_FP16, 2, 64, 1)
    a = dict(x=A, xs=0, heads=3, src=fs.FS_SRC_FP16, pos=A, n=5, inverse=0, out=A, os=0)
    assert L.fs_rope(pool, m, *{**a, **bad}.values(), None) == fs.FS_ERR_INVALID
    assert L.fs_rope(pool, -1, *a.values(), None) == fs.FS_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(new=0), dict(n_seq=0), dict(ids=0), dict(n_ids=-1), dict(tables=0), dict(max_blocks=0), dict(lens=0), dict(off=0),
                                 dict(seq=0), dict(pos=0), dict(n=-1), dict(n=1 << 31), dict(n_seq=1 << 30), dict(n_ids=1 << 31)])
def test_batch_tables_refusals(pool, bad):
    L = fs.binding._L
    _, m = fs.fs_model_register(pool, fs.FS_KV_FP16, 2, 64, 1)
    a = dict(held=A, new=A, n_seq=3, ids=A, n_ids=4, tables=A, max_blocks=2, lens=A, off=A, seq=A, pos=A, slots=A, n=9, status=A)
    assert L.fs_batch_tables(pool, m, *{**a, **bad}.values(), None) == fs.FS_ERR_INVALID
    assert L.fs_batch_tables(pool, m + 1, *a.values(), None) == fs.FS_ERR_INVALID


# ------------------------------------------------------------------------------------------------ the plain implementations
def test_plain_e4m3():
    codes = np.arange(256)
    v = plain.e4m3_value(codes)
    assert v[0x7E] == 448 and v[0x01] == 2.0 ** -9 and v[0x38] == 1 and np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and v[0xB8] == -1
    fine = np.sort(np.unique(v[~np.isnan(v)]))
    mid = (fine[1:] + fine[:-1]) / 2
    for x in np.concatenate([fine, mid * (1 + 1e-12), mid * (1 - 1e-12)]):
        near = fine[np.argmin(np.abs(fine - x))]
        assert plain.e4m3_round(x) == near, x
    # ties go to the even code: 17 lies between 16 (0x58) and 18 (0x59), 19 between 18 and 20
    assert plain.e4m3_round(17.0) == 16 and plain.e4m3_round(19.0) == 20 and plain.e4m3_round(1e9) == 448


def test_plain_scale_exponent():
    for amax, e in ((448.0, 0), (448.0001, 1), (0.0, -15), (1e-30, -15), (1e30, 7), (1.0, -8), (0.875, -9), (0.876, -8), (57344.0, 7)):
        assert plain.scale_exponent(amax) == e, amax
        if e not in (-15, 7):
            assert amax <= 448 * 2.0 ** e and amax > 448 * 2.0 ** (e - 1)


def test_plain_tables():
    # blocks of 4: request 0 holds 6 (two blocks) and gets 3 (one further block), 1 gets nothing, 2 begins with 5 (two blocks)
    table = np.array([[9, 8, -5, -5], [7, -5, -5, -5], [-5, -5, -5, -5]])
    got = plain.tables([6, 1, 0], [3, 0, 5], [3, 4, 5, 6], table, 4, 10, 100)
    assert got["table"].tolist() == [[9, 8, 3, -5], [7, -5, -5, -5], [4, 5, -5, -5]] and got["status"] == 0
    assert got["seq_lens"].tolist() == [9, 1, 5] and got["q_offsets"].tolist() == [0, 3, 3, 8]
    assert got["seq_idx"].tolist() == [0, 0, 0, 2, 2, 2, 2, 2, -1, -1] and got["pos"].tolist() == [6, 7, 8, 0, 1, 2, 3, 4, -1, -1]
    assert got["slots"].tolist() == [34, 35, 12, 16, 17, 18, 19, 20, -1, -1]


def test_plain_rotation():
    y, _ = plain.rotate([[[1.0, 0.0, 5.0, 6.0]]], [1], np.array([np.pi / 2]), halves=False)
    np.testing.assert_allclose(y, [[[0, 1, 5, 6]]], atol=1e-15)
    y, _ = plain.rotate([[[1.0, 2.0, 3.0, 4.0]]], [2], np.array([np.pi / 2, np.pi / 4]), halves=True)
    np.testing.assert_allclose(y, [[[-1, -4, -3, 2]]], atol=1e-14)
