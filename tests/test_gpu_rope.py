"""fs_rope and fs_rope_append: against the rotation in 64 bits, and the append's bytes against fs_kv_append of rotated fp32 keys."""
import numpy as np
import pytest

import block_cache as plain
import paper_2509_06261_amd as fs

pytestmark = pytest.mark.gpu

# An element is a cos + b sin times the amplitude: cosine and sine off by at most 2e-7 (the angle 5e-8, the series 2.5e-8, their
# roundings), two roundings to fp32 of 6e-8 each.
COMPUTE = 3e-7
HALF_STEP = dict(fp16=2.0 ** -11, fp32=2.0 ** -24)
TINY = dict(fp16=2.0 ** -25, fp32=0.0)  # half the spacing of subnormals


def make_model(d, kind=fs.FS_KV_FP16, heads=1, t=16, layers=1, n_blocks=1):
    import torch
    block = fs.fs_block_bytes(kind, heads, d, layers, t)
    mem = torch.zeros(n_blocks * block, dtype=torch.uint8, device="cuda")
    pool = fs.fs_pool_create(block, n_blocks * block, mem)
    return pool, fs.fs_model_register_tokens(pool, kind, heads, d, layers, t)[1], mem


def check_rotated(got, x, pos, f, halves, src, amplitude=1.0, inverse=False, from_fp32=False):
    """src: the type of `got`; from_fp32: x was of another, so that elements that are not rotated are rounded too (half a step)."""
    want, m = plain.rotate(x, pos, f, halves, amplitude, inverse)
    off = np.abs(got - want)
    tol = COMPUTE * m + HALF_STEP[src] * np.abs(want) * 1.01 + TINY[src]
    if not from_fp32:
        tol[..., 2 * len(f):] = 0
    assert (off <= tol).all(), (off - tol).max()


@pytest.mark.parametrize("src", ["fp16", "fp32"])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("d,r", [(8, 8), (8, 2), (16, 12), (64, 64), (64, 32), (64, 20), (128, 128), (128, 96), (128, 126), (128, 16), (256, 256), (512, 512), (512, 130)])
def test_rotation(d, r, halves, src):
    import torch
    rng = np.random.default_rng([d, r])
    pool, m, mem = make_model(d)
    fs.fs_model_set_rope(pool, m, fs.make_rope(r, 10000.0, layout=fs.FS_ROPE_HALVES if halves else fs.FS_ROPE_PAIRS))
    f = plain.frequencies(r, 10000.0, "none")
    dt = torch.float16 if src == "fp16" else torch.float32
    for n, heads, wide in ((1, 1, 0), (3, 5, 0), (67, 3, 40), (301, 33, 8)):
        rows = torch.from_numpy(rng.standard_normal((n, heads * d + wide)).astype(np.float32)).to("cuda", dt)
        x = rows[:, :heads * d].view(n, heads, d)
        pos = rng.integers(0, 5000, n)
        pos_d = torch.from_numpy(pos.astype(np.int32)).cuda()
        for inverse in (False, True):
            out = torch.full((n, heads, d), 9.0, dtype=dt, device="cuda")
            fs.fs_rope(pool, m, x, pos_d, out, inverse=inverse)
            check_rotated(out.double().cpu().numpy(), x.double().cpu().numpy(), pos, f, halves, src, inverse=inverse)
        keep = rows.clone()
        fs.fs_rope(pool, m, x, pos_d, x, inverse=True)  # in place, rows apart
        assert torch.equal(x, out) and torch.equal(rows[:, heads * d:], keep[:, heads * d:])
    fs.fs_pool_destroy(pool)


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "wavelength", "dimension"])
def test_far_positions_and_scaling(scaling):
    import torch
    par = dict(factor=8.0, low=1.0, high=32.0)
    pool, m, mem = make_model(128)
    kinds = dict(none=0, linear=1, base=2, wavelength=3, dimension=4)
    fs.fs_model_set_rope(pool, m, fs.make_rope(128, 500000.0, scaling=kinds[scaling], original_positions=4096, amplitude=1.25, **par))
    f = plain.frequencies(128, 500000.0, scaling, original=4096, **par)
    rng = np.random.default_rng(5)
    pos = np.concatenate([[0, 1, 2, 4095, 4096, 131071, 10 ** 6, 2 ** 24 + 1, 10 ** 8], rng.integers(0, 2 * 10 ** 6, 300)])
    x = rng.standard_normal((len(pos), 2, 128)).astype(np.float32)
    xd = torch.from_numpy(x).cuda()
    out = torch.empty_like(xd)
    fs.fs_rope(pool, m, xd, torch.from_numpy(pos.astype(np.int32)).cuda(), out)
    # (the 64-bit angles of the comparison are themselves off by pos * 2^-53)
    check_rotated(out.double().cpu().numpy(), x, pos, f, True, "fp32", amplitude=1.25)
    fs.fs_pool_destroy(pool)


def test_the_largest_position():
    """2^31 - 1 times a frequency that is a dyadic fraction of a turn: the angle is known exactly."""
    import torch
    pool, m, mem = make_model(8)
    rope = fs.make_rope(2, 2.0, scaling=fs.FS_ROPE_LINEAR, factor=8.0 / (2 * np.pi) / 1.0)  # f = 2 pi / 8 up to a double's rounding
    fs.fs_model_set_rope(pool, m, rope)
    f = float(fs.fs_rope_frequencies(rope)[0])
    x = torch.zeros((1, 1, 8), device="cuda")
    x[0, 0, 0] = 1.0
    out = torch.empty_like(x)
    p = 2 ** 31 - 1
    fs.fs_rope(pool, m, x, torch.tensor([p], dtype=torch.int32, device="cuda"), out)
    from fractions import Fraction
    # the angle from exact products of doubles; 2 pi to 60 digits
    two_pi = Fraction("6.283185307179586476925286766559005768394338798750211641949889")
    turns = Fraction(f) * p / two_pi
    frac = float(turns - int(turns)) * 2 * np.pi
    # (the double f is within 2^-54 of the long double that is used: 2^31 of them are 2e-7 radians)
    np.testing.assert_allclose(out[0, 0, :2].double().cpu().numpy(), [np.cos(frac), np.sin(frac)], atol=COMPUTE + 2.0 ** 31 * 2.0 ** -54 * 2)
    fs.fs_pool_destroy(pool)


def test_padding_infinities_and_what_is_not_rotated():
    import torch
    pool, m, mem = make_model(64)
    fs.fs_model_set_rope(pool, m, fs.make_rope(32, 10000.0))
    x = torch.randn((9, 2, 64), device="cuda", dtype=torch.float16)
    x[:, :, 40] = float("inf")
    x[:, :, 41] = float("nan")
    x[4, 1, 3] = float("inf")  # reaches its pair and nothing else
    pos = torch.tensor([0, 1, -1, 3, 4, -2 ** 31, 6, 7, 8], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 5.0)
    fs.fs_rope(pool, m, x, pos, out)
    assert (out[2] == 5).all() and (out[5] == 5).all()
    live = [0, 1, 3, 4, 6, 7, 8]
    assert torch.equal(out[live][:, :, 32:].view(torch.int16), x[live][:, :, 32:].view(torch.int16))  # bit by bit, NaN too
    bad = ~torch.isfinite(out[live][:, :, :32])
    assert {tuple(i) for i in bad.nonzero().tolist()} <= {(3, 1, 3), (3, 1, 19)} and bad.any()
    assert torch.equal(out[0, :, :32], x[0, :, :32])  # position 0
    fs.fs_rope(pool, m, x[:0], pos[:0], out[:0])  # no tokens
    fs.fs_pool_destroy(pool)


def test_gradient_is_the_inverse():
    """d/dx <w, rope(x)> is fs_rope(w, inverse): against the definition's matrix and against differences, in fp32."""
    import torch
    rng = np.random.default_rng(3)
    for halves in (True, False):
        pool, m, mem = make_model(16)
        fs.fs_model_set_rope(pool, m, fs.make_rope(12, 100.0, layout=int(not halves), amplitude=1.5))
        f = plain.frequencies(12, 100.0, "none")
        n = 7
        x, w = (torch.from_numpy(rng.standard_normal((n, 2, 16)).astype(np.float32)).cuda() for _ in range(2))
        pos = torch.arange(n, dtype=torch.int32, device="cuda") * 11
        grad = torch.empty_like(w)
        fs.fs_rope(pool, m, w, pos, grad, inverse=True)
        check_rotated(grad.double().cpu().numpy(), w.cpu().numpy(), pos.cpu().numpy(), f, halves, "fp32", amplitude=1.5, inverse=True)

        def loss(x):
            y = torch.empty_like(x)
            fs.fs_rope(pool, m, x, pos, y)
            return (w.double() * y.double()).sum((1, 2)).cpu().numpy()

        for i in range(16):  # the map is linear: a difference of any size is the derivative, up to roundings of 16 products
            e = torch.zeros_like(x)
            e[:, 1, i] = 4.0
            diff = (loss(x + e) - loss(x - e)) / 8.0
            np.testing.assert_allclose(diff, grad[:, 1, i].double().cpu().numpy(), atol=32 * 2.0 ** -24 * 8 * 4)
        fs.fs_pool_destroy(pool)


# ------------------------------------------------------------------------------------------------------- fs_rope_append
KINDS = dict(fp16=fs.FS_KV_FP16, fp8=fs.FS_KV_FP8_E4M3, int8=fs.FS_KV_INT8, int4=fs.FS_KV_INT4, block=fs.FS_KV_FP8_BLOCK)


class Cache:
    def __init__(self, kind, heads, d, t, layers, lens, seed, rope):
        import torch
        rng = np.random.default_rng(seed)
        blocks = -(-np.asarray(lens) // t)
        n = int(blocks.sum()) + 3
        self.pool, self.model, self.mem = make_model(d, KINDS[kind], heads, t, layers, n)
        if kind == "fp8":
            k = rng.uniform(0.004, 0.02, (2, layers, heads))
            fs.fs_model_set_fp8_scales(self.pool, self.model, k[0], k[1])
        fs.fs_model_set_rope(self.pool, self.model, rope)
        ids = rng.permutation(n)
        table, at = np.full((len(lens), int(blocks.max())), -1), 0
        for i, b in enumerate(blocks):
            table[i, :b] = ids[at:at + b]
            at += b
        self.table = torch.from_numpy(table.astype(np.int32)).cuda()

    def close(self):
        fs.fs_pool_destroy(self.pool)


def new_tokens(lens, held=None):
    held = np.zeros_like(lens) if held is None else held
    seq = np.repeat(np.arange(len(lens)), lens - held)
    pos = np.concatenate([np.arange(h, n) for h, n in zip(held, lens)])
    return seq.astype(np.int32), pos.astype(np.int32)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("src", ["fp16", "fp32"])
@pytest.mark.parametrize("heads,group,d,t,r,halves,wide,lens", [
    (2, 4, 128, 16, 128, True, True, [1, 40, 17, 3]), (3, 1, 64, 9, 32, False, False, [70, 1, 64]), (1, 2, 8, 5, 6, True, False, [11, 12]),
    (8, 4, 128, 63, 96, True, True, [500, 700, 1, 129, 2000]), (2, 8, 256, 33, 256, False, True, [100, 31]), (1, 1, 512, 3, 100, True, True, [20]),
    (5, 3, 16, 130, 10, True, True, [300, 130, 260])])
def test_append_equals_rope_then_append(kind, src, heads, group, d, t, r, halves, wide, lens):
    import torch
    lens = np.array(lens)
    rope = fs.make_rope(r, 10000.0, layout=int(not halves), amplitude=1.0)
    a, b = (Cache(kind, heads, d, t, 2, lens, 7, rope) for _ in range(2))
    dt = torch.float16 if src == "fp16" else torch.float32
    rng = np.random.default_rng(11)
    held = np.zeros_like(lens)
    for part in range(2):  # a prefix of every sequence, then the rest
        upto = np.maximum(lens // 2, 1) if part == 0 else lens
        seq, pos = (torch.from_numpy(x).cuda() for x in new_tokens(upto, held))
        held = upto
        n, nq = len(seq), heads * group
        if n == 0:
            continue
        qkv = torch.from_numpy((rng.standard_normal((n, (nq + 2 * heads) * d)) * (1 + part * 3)).astype(np.float32)).to("cuda", dt)
        q, k, v = ((x if wide else x.contiguous()).view(n, -1, d) for x in qkv.split([nq * d, heads * d, heads * d], dim=1))
        q_out = torch.full((n, nq, d), 7.0, dtype=torch.float16, device="cuda")
        fs.fs_rope_append(a.pool, a.model, 1, q, k, v, seq, pos, a.table, q_out)
        k32 = torch.empty((n, heads, d), device="cuda")
        fs.fs_rope(b.pool, b.model, k.float().contiguous(), pos, k32)
        fs.fs_kv_append(b.pool, b.model, 1, k32, v.float().contiguous(), seq, pos, b.table)
        assert torch.equal(a.mem, b.mem)
        check_rotated(q_out.double().cpu().numpy(), q.double().cpu().numpy(), pos.cpu().numpy(), plain.frequencies(r, 10000.0, "none"), halves, "fp16", from_fp32=src == "fp32")
    a.close()
    b.close()


@pytest.mark.parametrize("kind", list(KINDS))
def test_padding_and_tokens_without_a_block(kind):
    import torch
    lens = np.array([40, 40])
    c = Cache(kind, 2, 64, 16, 1, lens, 3, fs.make_rope(64, 10000.0))
    n = 70
    q, k, v = (torch.randn((n, h, 64), device="cuda", dtype=torch.float16) for h in (4, 2, 2))
    seq = torch.zeros(n, dtype=torch.int32, device="cuda")
    pos = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    # padding (-1, and the smallest int), a negative sequence, positions past the table, a table entry of no block
    pos[10:20] = torch.arange(10, dtype=torch.int32, device="cuda")
    pos[21] = -2 ** 31
    pos[30], seq[30] = 5, -1
    pos[31], pos[32] = 48, 2 ** 31 - 1
    pos[33], seq[33] = 17, 1
    c.table[1, 1] = 1 << 20
    q_out = torch.full((n, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    fs.fs_rope_append(c.pool, c.model, 0, q, k, v, seq, pos, c.table, q_out)
    written = {i for i in range(n) if (q_out[i] != 7).any()}
    assert written == set(range(10, 20)) | {30, 31, 32, 33}
    block = fs.fs_model_geometry(c.pool, c.model).block_budget
    touched = {i // block for i in c.mem.nonzero()[:, 0].tolist()}
    assert touched == {int(c.table[0, 0])}
    # keys and values alone; no tokens at all
    before = c.mem.clone()
    fs.fs_rope_append(c.pool, c.model, 0, None, k[10:20], v[10:20], seq[10:20], pos[10:20], c.table, None)
    assert torch.equal(c.mem, before)
    fs.fs_rope_append(c.pool, c.model, 0, q[:0], k[:0], v[:0], seq[:0], pos[:0], c.table, q_out[:0])
    c.close()


def both_appends(kind, src, heads, group, d, t, rope, lens, pads, seed):
    """One call, and fs_rope with fs_kv_append: the same bytes and the same queries.  Returns q, q_out, positions."""
    import torch
    lens = np.array(lens)
    a, b = (Cache(kind, heads, d, t, 2, lens, 7, rope) for _ in range(2))
    rng = np.random.default_rng(seed)
    dt = torch.float16 if src == "fp16" else torch.float32
    held = np.zeros_like(lens)
    for upto in (np.maximum(lens // 40, 1), lens):  # few tokens, then the many
        seq, pos = new_tokens(upto, held)
        held = upto
        if pads:  # behind every sequence a few tokens of nobody
            cuts = np.cumsum(np.unique(seq, return_counts=True)[1])
            seq, pos = (np.insert(x, np.repeat(cuts, pads), f) for x, f in ((seq, 0), (pos, -1)))
        seq, pos = torch.from_numpy(seq).cuda(), torch.from_numpy(pos).cuda()
        n, nq = len(seq), heads * group
        qkv = (torch.randn((n, (nq + 2 * heads) * d), device="cuda", generator=torch.Generator("cuda").manual_seed(seed)) * 2).to(dt)
        q, k, v = (x.view(n, -1, d) for x in qkv.split([nq * d, heads * d, heads * d], dim=1))
        q_out, q_ref = (torch.full((n, nq, d), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
        fs.fs_rope_append(a.pool, a.model, 1, q, k, v, seq, pos, a.table, q_out)
        k32, q32 = torch.zeros((n, heads, d), device="cuda"), torch.zeros((n, nq, d), device="cuda")
        fs.fs_rope(b.pool, b.model, k.float().contiguous(), pos, k32)
        fs.fs_kv_append(b.pool, b.model, 1, k32, v.float().contiguous(), seq, pos, b.table)
        fs.fs_rope(b.pool, b.model, q.float().contiguous(), pos, q32)
        q_ref[pos >= 0] = q32[pos >= 0].half()
        assert torch.equal(a.mem, b.mem)
        assert torch.equal(q_out, q_ref)
    a.close()
    b.close()
    return q, q_out, pos


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("src", ["fp16", "fp32"])
@pytest.mark.parametrize("r,halves", [(64, True), (64, False), (42, True)])
def test_prompts_of_many_tokens(kind, src, r, halves):
    """More rows than the card has waves: the queries go by themselves, and FP8_BLOCK's groups are cut differently."""
    q, q_out, pos = both_appends(kind, src, 8, 4, 64, 17, fs.make_rope(r, 10000.0, layout=int(not halves)), [5000, 4400, 1, 16, 18], 3, 2)
    some = np.random.default_rng(1).permutation(np.flatnonzero(pos.cpu().numpy() >= 0))[:50]
    check_rotated(q_out[some].double().cpu().numpy(), q[some].double().cpu().numpy(), pos.cpu().numpy()[some], plain.frequencies(r, 10000.0, "none"), halves, "fp16", from_fp32=src == "fp32")


@pytest.mark.parametrize("src", ["fp16", "fp32"])
@pytest.mark.parametrize("heads,group,d,t,r,halves,lens", [
    (2, 2, 256, 100, 256, True, [200, 199, 5]), (3, 1, 128, 200, 128, False, [1000, 201]), (1, 8, 512, 70, 100, True, [140, 3]), (2, 1, 64, 400, 22, True, [900, 400, 401]),
    (1, 1, 128, 200, 128, True, [9000, 100])])
def test_blocks_of_more_rows_than_fit_in_registers(src, heads, group, d, t, r, halves, lens):
    both_appends("block", src, heads, group, d, t, fs.make_rope(r, 10000.0, layout=int(not halves)), lens, 0, 4)


def test_rotation_of_many_rows():
    """The launches whose waves take several rows: against the definition at rows drawn over all of them."""
    import torch
    rng = np.random.default_rng(6)
    for d, r, halves in ((128, 128, True), (64, 64, False), (128, 126, True)):
        pool, m, mem = make_model(d)
        fs.fs_model_set_rope(pool, m, fs.make_rope(r, 10000.0, layout=int(not halves)))
        for dt in (torch.float16, torch.float32):
            x = torch.randn((9001, 33, d), device="cuda").to(dt)
            pos = torch.from_numpy(rng.integers(0, 100000, 9001).astype(np.int32)).cuda()
            pos[77] = -1
            out = torch.full_like(x, 3.0)
            fs.fs_rope(pool, m, x, pos, out)
            assert (out[77] == 3).all()
            some = rng.permutation(9001)[:60]
            some = np.concatenate([some[some != 77], [0, 1, 8999, 9000]])
            check_rotated(out[some].double().cpu().numpy(), x[some].double().cpu().numpy(), pos.cpu().numpy()[some], plain.frequencies(r, 10000.0, "none"), halves, "fp16" if dt == torch.float16 else "fp32")
        fs.fs_pool_destroy(pool)


def test_rows_of_another_model_are_refused():
    """Also of one token, whose stride nobody needs."""
    import torch
    c = Cache("fp16", 2, 64, 16, 1, np.array([5]), 3, fs.make_rope(64, 10000.0))
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    for stream in (None, torch.cuda.current_stream().cuda_stream):  # natively and through ctypes
        def rows(h, d, n=1):
            return torch.ones((n, h, d), device="cuda", dtype=torch.float16)
        fs.fs_rope(c.pool, c.model, rows(3, 64), one, rows(3, 64), stream=stream)
        with pytest.raises(fs.FsError):
            fs.fs_rope(c.pool, c.model, rows(3, 32), one, rows(3, 32), stream=stream)
        fs.fs_rope_append(c.pool, c.model, 0, rows(4, 64), rows(2, 64), rows(2, 64), one, one, c.table, rows(4, 64), stream=stream)
        for q, kv in (((4, 32), (2, 64)), ((4, 64), (1, 64)), ((4, 64), (2, 32))):
            with pytest.raises(fs.FsError):
                fs.fs_rope_append(c.pool, c.model, 0, rows(*q), rows(*kv), rows(*kv), one, one, c.table, rows(*q), stream=stream)
    c.close()
