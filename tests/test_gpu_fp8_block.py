"""The FP8_BLOCK format: appended bytes, decode and prefill attention, against plain implementations in 64 bits."""
import math

import numpy as np
import pytest

import block_cache as plain
import paper_2509_06261_amd as fs

pytestmark = pytest.mark.gpu


class Cache:
    """A pool of FP8_BLOCK blocks, its tables dealt in random order; spare: blocks that belong to nobody."""

    def __init__(self, heads, d, t, lens, seed=0, layers=2, layer=1, spare=2, fill=True):
        import torch
        self.heads, self.d, self.t, self.layers, self.layer = heads, d, t, layers, layer
        self.lens = np.asarray(lens, np.int64)
        self.rng = np.random.default_rng(seed)
        blocks = -(-self.lens // t)
        self.n = int(blocks.sum()) + spare
        p = plain.layout(heads, d, t, layers)
        self.mem = torch.zeros(self.n * p["block"], dtype=torch.uint8, device="cuda")
        self.pool = fs.fs_pool_create(p["block"], self.mem.numel(), self.mem)
        _, self.model = fs.fs_model_register_tokens(self.pool, fs.FS_KV_FP8_BLOCK, heads, d, layers, t)
        ids, at = self.rng.permutation(self.n), 0
        self.table_host = np.full((len(lens), int(max(blocks.max(), 1))), -1)
        for i, b in enumerate(blocks):
            self.table_host[i, :b] = ids[at:at + b]
            at += b
        self.table = torch.from_numpy(self.table_host.astype(np.int32)).cuda()
        self.seq_lens = torch.from_numpy(self.lens.astype(np.int32)).cuda()
        if fill:
            self.k, self.v = plain.fill_random(self.mem, (heads, d, t, layers), layer, self.rng)
            self._spoil_dead_slots()

    def _spoil_dead_slots(self):
        """Slots past a sequence's end hold NaN codes, blocks of nobody NaN scales: neither may show."""
        import torch
        k, v, scales = plain.views(self.mem, self.heads, self.d, self.t, self.layers, self.layer)
        for i, n in enumerate(self.lens):
            if n % self.t:
                b = int(self.table_host[i, n // self.t])
                k[b, :, n % self.t:] = 0x7F
                v[b, :, n % self.t:] = 0xFF
        used = set(self.table_host[self.table_host >= 0].tolist())
        for b in set(range(self.n)) - used:
            scales[b] = torch.nan

    def rows(self, i, n):
        """K and V [n][heads][d] of sequence i."""
        at = np.arange(n)
        blk = self.table_host[i, at // self.t]
        return self.k[blk, :, at % self.t], self.v[blk, :, at % self.t]

    def queries(self, n, group):
        import torch
        q = self.rng.standard_normal((n, self.heads * group, self.d)) * np.linspace(0.3, 2.0, self.heads * group)[None, :, None]
        qd = torch.from_numpy(q.astype(np.float16)).cuda()
        return qd, qd.double().cpu().numpy()

    def close(self):
        fs.fs_pool_destroy(self.pool)


def compare(cache, out, lse, q, group, scale, rows):
    """rows: (row of q / out, sequence, tokens that it sees)."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r, i, n in rows:
        k, v = cache.rows(i, n)
        for h in range(cache.heads):
            g = slice(h * group, (h + 1) * group)
            want, want_lse, sum_abs = plain.attention(q[r, g], k[:, h], v[:, h], scale)
            tol = plain.out_tolerance(want, sum_abs, n, np.abs(v[:, h]).max())
            off = np.abs(out[r, g] - want)
            assert (off <= tol).all(), (r, i, n, h, (off / tol).max())
            # fp32 sums of d products and of n weights, base-2 exponentials
            assert np.abs(lse[r, g] - want_lse).max() <= 2e-5 + 2e-6 * np.abs(want_lse).max()


def decode(cache, group, scale, host=True, option=None, multi=True, status=0):
    import torch
    for o, value in (option or {}).items():
        assert fs.fs_pool_set_option(cache.pool, o, value) == fs.FS_OK
    q, qh = cache.queries(len(cache.lens), group)
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    b = fs.make_batch(cache.model, cache.layer, q.shape[1], scale, q, cache.table, cache.seq_lens, out, lse, cache.lens.astype(np.int32) if host else None)
    ws = torch.empty(fs.fs_decode_workspace_bytes(cache.pool, [b]), dtype=torch.uint8, device="cuda")
    if multi:
        fs.fs_decode_attention_multi(cache.pool, [b], ws)
    else:
        fs.fs_decode_attention(cache.pool, cache.model, cache.layer, q.shape[1], scale, q, cache.table, cache.seq_lens, out, lse, ws)
    assert fs.fs_decode_status(ws) == status
    return out, lse, qh


# ------------------------------------------------------------------------------------------------------------- decode
@pytest.mark.parametrize("kernel", ["automatic", "list", "generic", "split"])
@pytest.mark.parametrize("heads,group,d,t,lens", [
    (2, 4, 128, 16, [1, 15, 16, 17, 100, 333]), (1, 8, 128, 63, [64, 2000, 1, 63]), (3, 1, 64, 9, [9, 10, 257, 1]), (2, 16, 64, 31, [400, 31, 5]),
    (2, 5, 256, 33, [1, 90, 700]), (1, 2, 256, 8, [8, 64, 65]), (4, 4, 128, 127, [1500, 127, 128, 3])])
def test_decode(heads, group, d, t, lens, kernel):
    option = dict(automatic={}, list={fs.FS_OPT_DECODE_WORK_LIST: 1}, generic={fs.FS_OPT_DECODE_KERNEL: 1}, split={fs.FS_OPT_SPLIT_BYTES: 16384})[kernel]
    c = Cache(heads, d, t, lens)
    scale = 1 / math.sqrt(d)
    out, lse, q = decode(c, group, scale, host=kernel != "list", option=option, multi=kernel != "list")
    compare(c, out, lse, q, group, scale, [(i, i, int(n)) for i, n in enumerate(lens)])
    assert fs.fs_pool_get_option(c.pool, fs.FS_OPT_LAST_DECODE_KERNEL) == dict(automatic=4, list=2, generic=1, split=2)[kernel]
    c.close()


@pytest.mark.parametrize("heads,group,d,t,lens", [(2, 4, 32, 16, [1, 40, 300]), (1, 2, 512, 5, [77, 5]), (2, 3, 128, 7, [1, 7, 8, 100]), (3, 1, 8, 100, [250, 100])])
def test_decode_of_shapes_for_the_vector_alu(heads, group, d, t, lens):
    c = Cache(heads, d, t, lens)
    out, lse, q = decode(c, group, 0.2)
    compare(c, out, lse, q, group, 0.2, [(i, i, int(n)) for i, n in enumerate(lens)])
    c.close()


def test_long_sequences():
    lens = [32768, 9001, 1]
    c = Cache(1, 128, 126, lens, layers=1, layer=0)
    for host in (True, False):
        out, lse, q = decode(c, 8, 0.1, host=host)
        compare(c, out, lse, q, 8, 0.1, [(i, i, int(n)) for i, n in enumerate(lens)])
    c.close()


def test_extreme_scales():
    """Scales at both ends of their range: every value is still an fp16 number, subnormal ones included."""
    lens = [200, 64]
    for e_k, e_v in ((-15, -15), (7, -15), (-15, 7)):
        c = Cache(2, 128, 64, lens, seed=e_k + 40)
        k, v, scales = plain.views(c.mem, 2, 128, 64, 2, 1)
        for which, (e, rows) in enumerate(((e_k, c.k), (e_v, c.v))):
            old = 2.0 ** np.rint(np.log2(scales[:, :, which].double().cpu().numpy()))
            rows *= (2.0 ** e / old)[:, :, None, None]
            scales[:, :, which] = 2.0 ** e
        scale = 0.1 if e_k < 0 else 1e-6
        for kernel in (0, 1):
            out, lse, q = decode(c, 4, scale, option={fs.FS_OPT_DECODE_KERNEL: kernel})
            compare(c, out, lse, q, 4, scale, [(0, 0, 200), (1, 1, 64)])
        c.close()


def test_every_code_and_scale_converts_exactly():
    """One token per sequence: its output is its V row, so that all codes are seen under all scales."""
    import torch
    c = Cache(1, 256, 8, [1] * 23, layers=1, layer=0)
    _, v, scales = plain.views(c.mem, 1, 256, 8, 1, 0)
    codes = np.arange(256)
    want = []
    for i in range(23):
        b = int(c.table_host[i, 0])
        v[b, 0, 0] = torch.from_numpy(codes.astype(np.uint8)).cuda()
        v[b, 0, 0, 0x7F], v[b, 0, 0, 0xFF] = 0, 0
        scales[b, 0, 1] = 2.0 ** (i - 15)
        x = plain.e4m3_value(codes) * 2.0 ** (i - 15)
        x[[0x7F, 0xFF]] = 0
        want.append(x)
    for kernel in (0, 1):
        out, _, _ = decode(c, 4, 0.1, option={fs.FS_OPT_DECODE_KERNEL: kernel})
        assert (out.double().cpu().numpy() == np.array(want)[:, None]).all()
    c.close()


def test_beside_the_other_formats_in_one_launch():
    import torch
    rng = np.random.default_rng(9)
    slab = 1 << 17
    mem = torch.zeros(64 * slab, dtype=torch.uint8, device="cuda")
    pool = fs.fs_pool_create(slab, 64 * slab, mem)
    results = {}
    lens = np.array([1, 100, 333], np.int32)
    batches, keep, models = [], [], []
    for kind in (fs.FS_KV_FP16, fs.FS_KV_FP8_BLOCK, fs.FS_KV_INT8, fs.FS_KV_FP8_E4M3, fs.FS_KV_INT4):
        t, m = fs.fs_model_register(pool, kind, 2, 128, 1)
        if kind == fs.FS_KV_FP8_E4M3:
            fs.fs_model_set_fp8_scales(pool, m, np.full((1, 2), 0.02), np.full((1, 2), 0.02))
        table = np.zeros((3, -(-333 // t)), np.int32)
        for i, n in enumerate(lens):
            rc, table[i, :-(-n // t)] = fs.fs_blocks_alloc(pool, m, -(-int(n) // t))
            assert rc == 0
        table = torch.from_numpy(table).cuda()
        seq = torch.from_numpy(np.repeat(np.arange(3), lens).astype(np.int32)).cuda()
        pos = torch.from_numpy(np.concatenate([np.arange(n) for n in lens]).astype(np.int32)).cuda()
        k, v = (torch.from_numpy(rng.standard_normal((len(seq), 2, 128)).astype(np.float16)).cuda() for _ in range(2))
        q = torch.from_numpy(rng.standard_normal((3, 8, 128)).astype(np.float16)).cuda()
        out, lse = torch.zeros_like(q), torch.zeros((3, 8), device="cuda")
        lens_d = torch.from_numpy(lens).cuda()
        models.append((m, k, v, seq, pos, table, q))
        batches.append(fs.make_batch(m, 0, 8, 0.09, q, table, lens_d, out, lse, lens))
        keep.append((out, lse, lens_d))
    # the whole step in one call: all tokens appended by the front kernel, then attention
    ws = torch.empty(fs.fs_decode_workspace_bytes(pool, batches), dtype=torch.uint8, device="cuda")
    for work_list in (0, 1):
        assert fs.fs_pool_set_option(pool, fs.FS_OPT_DECODE_WORK_LIST, work_list) == 0
        mem.zero_()
        appends = [fs.make_append(m, 0, k, v, seq, pos, table) for m, k, v, seq, pos, table, _ in models]
        fs.fs_decode_step_multi(pool, appends, batches, ws)
        assert fs.fs_decode_status(ws) == 0
        results[work_list] = [(o.clone(), s.clone()) for o, s, _ in keep]
        # the same bytes as by appends of their own
        stepped = mem.clone()
        mem.zero_()
        for m, k, v, seq, pos, table, _ in models:
            fs.fs_kv_append(pool, m, 0, k, v, seq, pos, table)
        assert torch.equal(mem, stepped)
        mem.zero_()
        fs.fs_kv_append_multi(pool, appends)
        assert torch.equal(mem, stepped)
    for work_list in (0, 1):
        for (m, k, v, seq, pos, table, q), (out, lse) in zip(models, results[work_list]):
            for i, n in enumerate(lens):
                ki, vi = (x[seq == i].double().cpu().numpy() for x in (k, v))
                for h in range(2):
                    want, _, sum_abs = plain.attention(q[i, 4 * h:4 * h + 4].double().cpu().numpy(), ki[:, h], vi[:, h], 0.09)
                    # (the formats' own roundings: half a step of 4 bits over a range of 9, of the keys and of the values)
                    assert np.abs(out[i, 4 * h:4 * h + 4].double().cpu().numpy() - want).max() < 1.0
    # attention over FP8_BLOCK beside the others is what it is alone
    out, lse = (torch.zeros_like(x) for x in keep[1][:2])
    m, _, _, _, _, table, q = models[1]
    alone = fs.make_batch(m, 0, 8, 0.09, q, table, keep[1][2], out, lse, lens)
    ws2 = torch.empty(fs.fs_decode_workspace_bytes(pool, [alone]), dtype=torch.uint8, device="cuda")
    fs.fs_decode_attention_multi(pool, [alone], ws2)
    torch.testing.assert_close(out, results[1][1][0], rtol=4e-3, atol=4e-3)
    fs.fs_pool_destroy(pool)


def test_bad_lengths_and_blocks_are_reported():
    c = Cache(2, 128, 16, [40, 50])
    c.table[0, 1] = 1 << 20
    out, lse, q = decode(c, 4, 0.1, status=4)
    compare(c, out, lse, q, 4, 0.1, [(1, 1, 50)])
    c.table[0, 1] = int(c.table_host[0, 1])
    c.seq_lens[0] = 1000  # (clamped to the table's four blocks, the fourth of which names none)
    out, lse, q = decode(c, 4, 0.1, host=False, status=5)
    compare(c, out, lse, q, 4, 0.1, [(1, 1, 50)])
    c.close()


def test_blocks_beyond_four_gigabytes():
    import torch
    p = plain.layout(2, 128, 64, 1)
    n = (5 << 30) // p["block"]
    mem = torch.empty(n * p["block"], dtype=torch.uint8, device="cuda")
    pool = fs.fs_pool_create(p["block"], mem.numel(), mem)
    _, m = fs.fs_model_register_tokens(pool, fs.FS_KV_FP8_BLOCK, 2, 128, 1, 64)
    ids = np.array([[n - 1, n // 2, n - 3]])
    rng = np.random.default_rng(2)
    lens = torch.tensor([150], dtype=torch.int32, device="cuda")
    k, v = (rng.standard_normal((150, 2, 128)).astype(np.float16) for _ in range(2))
    seq, pos = torch.zeros(150, dtype=torch.int32, device="cuda"), torch.arange(150, dtype=torch.int32, device="cuda")
    table = torch.from_numpy(ids.astype(np.int32)).cuda()
    fs.fs_kv_append(pool, m, 0, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), seq, pos, table)
    want = [plain.BlockCache(3, 2, 64, 128) for _ in range(2)]
    for w, x in zip(want, (k, v)):
        w.append(x.astype(np.float64), np.arange(150) // 64, np.arange(150) % 64)
    got_k, got_v, scales = plain.views(mem, 2, 128, 64, 1, 0)
    for i, b in enumerate(ids[0]):
        for w, rows, which in ((want[0], got_k, 0), (want[1], got_v, 1)):
            assert (scales[b, :, which].cpu().numpy() == 2.0 ** w.e[i]).all()
            assert (plain.e4m3_value(rows[b, :, :w.used[i]].cpu().numpy()) == w.codes[i][:, :w.used[i]]).all()
    q = torch.from_numpy(rng.standard_normal((1, 8, 128)).astype(np.float16)).cuda()
    out, lse = torch.zeros_like(q), torch.zeros((1, 8), device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    fs.fs_decode_attention(pool, m, 0, 8, 0.1, q, table, lens, out, lse, ws)
    for h in range(2):
        kk, vv = (np.concatenate([w.codes[i, h, :w.used[i]] * 2.0 ** w.e[i, h] for i in range(3)]) for w in want)
        x, _, s = plain.attention(q[0, 4 * h:4 * h + 4].double().cpu().numpy(), kk, vv, 0.1)
        assert (np.abs(out[0, 4 * h:4 * h + 4].double().cpu().numpy() - x) <= plain.out_tolerance(x, s, 150, np.abs(vv).max())).all()
    fs.fs_pool_destroy(pool)


# ------------------------------------------------------------------------------------------------------------- append
def append_parts(c, parts, src, make):
    """Appends the parts (lists of (sequence, first, end)) call by call; returns the plain caches of K and V."""
    import torch
    want = [plain.BlockCache(c.n, c.heads, c.t, c.d) for _ in range(2)]
    for part in parts:
        seq = np.concatenate([np.full(b - a, i) for i, a, b in part])
        pos = np.concatenate([np.arange(a, b) for _, a, b in part])
        rows = [make(len(seq)).astype(np.float16 if src == "fp16" else np.float32) for _ in range(2)]
        k, v = (torch.from_numpy(x).cuda() for x in rows)
        fs.fs_kv_append(c.pool, c.model, c.layer, k, v, torch.from_numpy(seq.astype(np.int32)).cuda(), torch.from_numpy(pos.astype(np.int32)).cuda(), c.table)
        blk, slot = c.table_host[seq, pos // c.t], pos % c.t
        for w, x in zip(want, rows):
            w.append(x.astype(np.float64), blk, slot)
    return want


def check_bytes(c, want):
    k, v, scales = plain.views(c.mem, c.heads, c.d, c.t, c.layers, c.layer)
    for which, (w, rows) in enumerate(zip(want, (k, v))):
        got = plain.e4m3_value(rows.cpu().numpy())
        sc = scales[:, :, which].double().cpu().numpy()
        for b in np.flatnonzero(w.used):
            assert (sc[b] == 2.0 ** w.e[b]).all(), (b, sc[b], w.e[b])
            assert np.array_equal(got[b, :, :w.used[b]], w.codes[b][:, :w.used[b]]), b
    if c.layers > 1:  # the other layers' bytes stay
        p = plain.layout(c.heads, c.d, c.t, c.layers)
        other = c.mem.view(c.n, c.layers, p["layer"])
        assert not other[:, [x for x in range(c.layers) if x != c.layer]].any()


@pytest.mark.parametrize("src", ["fp16", "fp32"])
@pytest.mark.parametrize("heads,d,t,lens", [(8, 128, 63, [1000, 64, 63, 1, 500]), (1, 64, 16, [100, 16]), (3, 8, 5, [23, 5, 6]), (2, 512, 7, [30]),
                                            (2, 256, 200, [601, 199]), (40, 128, 9, [40, 9]), (2, 32, 130, [400])])
def test_appended_bytes(heads, d, t, lens, src):
    """Whole prompts; then token by token and in chunks, rows growing from call to call so that scales grow."""
    for how in ("prompt", "token", "chunk"):
        c = Cache(heads, d, t, lens, fill=False)
        rng = np.random.default_rng(len(lens))
        size = [0.01]

        def make(n):
            size[0] *= 1.0 if how == "prompt" else 1.15
            x = rng.standard_normal((n, heads, d)) * min(size[0], 3000.0)
            x[rng.random(x.shape) < 0.05] = 0
            return x

        if how == "prompt":
            parts = [[(i, 0, n) for i, n in enumerate(lens)]]
        elif how == "token":
            parts = [[(i, p, p + 1) for i, n in enumerate(lens) if p < n] for p in range(min(max(lens), 70))]
        else:
            cut = [sorted({0, n, *rng.integers(0, n + 1, 4).tolist()}) for n in lens]
            parts = [[(i, s[k], s[k + 1]) for i, s in enumerate(cut) if k + 1 < len(s)] for k in range(max(map(len, cut)) - 1)]
        check_bytes(c, append_parts(c, parts, src, make))
        c.close()


def test_extreme_rows():
    """Zeros, values beyond the format, infinities and NaN (which become the largest magnitude), subnormal fp32 rows."""
    import torch
    c = Cache(1, 64, 8, [8, 8, 8, 8, 8, 8], fill=False)
    rows = np.zeros((6, 64), np.float32)
    rows[1] = 3e38
    rows[2, 5], rows[2, 6], rows[2, 7] = np.inf, -np.inf, np.nan
    rows[3] = 1e-40
    rows[4] = -np.float32(448) * np.float32(2.0) ** -15
    rows[5] = 57344.0 * 1.01
    x = torch.from_numpy(rows.reshape(6, 1, 64)).cuda()
    seq, pos = torch.arange(6, dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    fs.fs_kv_append(c.pool, c.model, 1, x, x, seq, pos, c.table)
    k, v, scales = plain.views(c.mem, 1, 64, 8, 2, 1)
    for i, (e, values) in enumerate([(-15, 0.0), (7, 448.0), (7, None), (-15, 0.0), (-15, -448.0), (7, 448.0)]):
        b = int(c.table_host[i, 0])
        assert (scales[b] == 2.0 ** e).all(), i
        got = plain.e4m3_value(k[b, 0, 0].cpu().numpy())
        if values is None:
            assert got[5] == 448 and got[6] == -448 and abs(got[7]) == 448 and not got[8:].any()
        else:
            assert (got == values).all()
        assert torch.equal(k[b], v[b])
    c.close()


def test_a_block_that_begins_anew_forgets_its_scale():
    import torch
    c = Cache(2, 128, 16, [16], fill=False)
    big, small = (np.random.default_rng(i).standard_normal((16, 2, 128)) * s for i, s in ((0, 1000.0), (1, 0.01)))
    for rows in (big, small):
        x = torch.from_numpy(rows.astype(np.float32)).cuda()
        i = torch.zeros(16, dtype=torch.int32, device="cuda")
        fs.fs_kv_append(c.pool, c.model, 1, x, x, i, torch.arange(16, dtype=torch.int32, device="cuda"), c.table)
    want = plain.BlockCache(c.n, 2, 16, 128)
    want.append(small.astype(np.float32).astype(np.float64), np.full(16, c.table_host[0, 0]), np.arange(16))
    check_bytes(c, [want, want])
    # garbage where the scale should be (a block whose first slot was never appended): the scale is taken into the range
    _, _, scales = plain.views(c.mem, 2, 128, 16, 2, 1)
    scales[int(c.table_host[0, 0])] = float("nan")
    x = torch.ones((1, 2, 128), device="cuda")
    fs.fs_kv_append(c.pool, c.model, 1, x, x, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((1,), 3, dtype=torch.int32, device="cuda"), c.table)
    assert (scales[int(c.table_host[0, 0])] == 2.0 ** 7).all()
    c.close()


def test_append_skips_what_has_no_place():
    import torch
    c = Cache(2, 64, 16, [40], fill=False)
    c.table[0, 2] = 1 << 24
    seq = torch.tensor([0, 0, -1, 0, 0, 0, 0, 0], dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 1, 2, -1, 40, 48, 2 ** 31 - 1, 16], dtype=torch.int32, device="cuda")
    x = torch.ones((8, 2, 64), device="cuda", dtype=torch.float16)
    fs.fs_kv_append(c.pool, c.model, 1, x, x, seq, pos, c.table)
    k, v, scales = plain.views(c.mem, 2, 64, 16, 2, 1)
    written = {(b, s) for b, _, s, _ in k.nonzero().tolist()}
    assert written == {(int(c.table_host[0, 0]), 0), (int(c.table_host[0, 0]), 1), (int(c.table_host[0, 1]), 0)}
    fs.fs_kv_append(c.pool, c.model, 1, x[:0], x[:0], seq[:0], pos[:0], c.table)
    c.close()


def test_slots_in_the_middle_are_written_again():
    """A block's other slots, in front and behind, keep their values when the new rows are larger."""
    c = Cache(3, 128, 64, [64, 200], fill=False)
    rng = np.random.default_rng(4)
    size = [1.0]

    def make(n):
        size[0] *= 5
        return rng.standard_normal((n, 3, 128)) * size[0]

    check_bytes(c, append_parts(c, [[(0, 0, 64), (1, 0, 200)], [(0, 20, 21), (1, 70, 90)], [(0, 63, 64), (1, 130, 150)], [(0, 1, 63), (1, 199, 200)]], "fp32", make))
    c.close()


def test_many_tokens_of_many_sequences():
    """Enough tokens that a unit looks for groups among 64 neighbours, groups of one token to several blocks."""
    rng = np.random.default_rng(1)
    lens = np.concatenate([np.ones(3000, np.int64), rng.integers(1, 300, 200), [5000]])
    rng.shuffle(lens)
    c = Cache(4, 64, 48, lens, layers=1, layer=0, fill=False)
    check_bytes(c, append_parts(c, [[(i, 0, int(n)) for i, n in enumerate(lens)]], "fp16", lambda n: rng.standard_normal((n, 4, 64))))
    c.close()


# ------------------------------------------------------------------------------------------------------------ prefill
def prefill(c, group, scale, new, option=None, least=False, status=0):
    import torch
    for o, value in (option or {}).items():
        assert fs.fs_pool_set_option(c.pool, o, value) == fs.FS_OK
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q, qh = c.queries(int(off[-1]), group)
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    n = len(new)
    ws = torch.empty((fs.fs_prefill_least_workspace_bytes if least else fs.fs_prefill_workspace_bytes)(n), dtype=torch.uint8, device="cuda")
    fs.fs_prefill_attention(c.pool, c.model, c.layer, q.shape[1], scale, q, c.table, c.seq_lens, torch.from_numpy(off).cuda(), off, out, lse, ws)
    assert fs.fs_decode_status(ws) == status
    assert not out.isnan().any() and not lse.isnan().any()
    return out, lse, qh, off


def some_rows(c, off, new, rng, most=40):
    rows = [(int(off[i] + r), i, int(c.lens[i] - new[i] + r + 1)) for i in range(len(new)) for r in range(int(new[i]))]
    ends = [rows[int(off[i]) + r] for i in range(len(new)) if new[i] for r in (0, int(new[i]) - 1)]
    return ends + [rows[i] for i in rng.choice(len(rows), min(most, len(rows)), replace=False)]


@pytest.mark.parametrize("heads,group,d,t,lens,new", [
    (2, 4, 128, 16, [100, 1, 333], [100, 1, 200]),           # small launches: items of 8 blocks
    (8, 4, 128, 63, [600, 1000, 64, 700], [600, 900, 64, 1]),  # and larger ones, ragged
    (8, 4, 128, 31, [2500, 3000], [200, 100]),               # chunks behind contexts: groups of waves
    (8, 4, 128, 64, [9000], [512]),                          # a long context, split among workgroups
    (8, 8, 128, 127, [700] * 12, [700] * 12),                # many items per unit: the queue
    (8, 4, 64, 50, [300, 900, 20], [300, 900, 20]),
    (8, 4, 64, 9, [1500] * 20, [1500] * 20),                 # wide items
    (1, 2, 64, 8, [30, 8], [30, 3]),                         # the 16-column kernel
    (2, 4, 256, 33, [500, 40], [500, 40]),
    (4, 4, 256, 16, [1200, 700, 300], [1200, 700, 300]),
    (40, 1, 128, 9, [200, 77], [150, 77]),
    (2, 16, 128, 8, [90, 300], [90, 10]),
    (2, 3, 32, 10, [40, 25], [40, 5]),                       # the vector ALU
    (1, 4, 128, 5, [23, 60], [23, 7]),
])
def test_prefill(heads, group, d, t, lens, new):
    c = Cache(heads, d, t, lens)
    scale = 1 / math.sqrt(d)
    out, lse, q, off = prefill(c, group, scale, new)
    rows = some_rows(c, off, new, c.rng)
    compare(c, out, lse, q, group, scale, rows)
    kernel = fs.fs_pool_get_option(c.pool, fs.FS_OPT_LAST_PREFILL_KERNEL)
    # options about kernels that this format has not do not change the call
    again, _, q2, _ = prefill(c, group, scale, new, option={fs.FS_OPT_PREFILL_COLUMN_BLOCKS: 4, fs.FS_OPT_PREFILL_WAVES: 4, fs.FS_OPT_PREFILL_PIPELINED: 1}, least=True)
    assert fs.fs_pool_get_option(c.pool, fs.FS_OPT_LAST_PREFILL_KERNEL) == kernel
    compare_out_only(c, again, q2, group, scale, rows[:8])
    c.close()


@pytest.mark.parametrize("heads,group,d,t,lens,new", [
    (2, 4, 128, 5, [5000, 2500, 2432], [100, 60, 1]), (1, 8, 64, 8, [9000, 8193], [300, 2]), (2, 4, 256, 3, [3300, 1409], [40, 9]), (8, 4, 128, 16, [9000, 8192], [400, 300]),
    (8, 4, 128, 7, [3700] * 9, [260] * 9)])
def test_prefill_of_more_blocks_than_a_table_holds(heads, group, d, t, lens, new):
    c = Cache(heads, d, t, lens)
    out, lse, q, off = prefill(c, group, 0.07, new)
    compare(c, out, lse, q, group, 0.07, some_rows(c, off, new, c.rng, most=10))
    c.close()


def compare_out_only(c, out, q, group, scale, rows):
    out = out.double().cpu().numpy()
    for r, i, n in rows:
        k, v = c.rows(i, n)
        for h in range(c.heads):
            g = slice(h * group, (h + 1) * group)
            want, _, sum_abs = plain.attention(q[r, g], k[:, h], v[:, h], scale)
            assert (np.abs(out[r, g] - want) <= plain.out_tolerance(want, sum_abs, n, np.abs(v[:, h]).max())).all()


def test_prefill_of_a_scale_that_is_not_positive():
    c = Cache(2, 128, 16, [100, 50])
    for scale in (0.0, -0.05):
        out, lse, q, off = prefill(c, 4, scale, [100, 20])
        compare(c, out, lse, q, 4, scale, some_rows(c, off, [100, 20], c.rng))
    c.close()


def test_prefill_reports_bad_blocks():
    c = Cache(2, 128, 16, [100, 50])
    c.table[1, 1] = -5
    import torch
    off = np.array([0, 100, 150], np.int32)
    q, qh = c.queries(150, 4)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.empty(fs.fs_prefill_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    fs.fs_prefill_attention(c.pool, c.model, 1, 8, 0.1, q, c.table, c.seq_lens, torch.from_numpy(off).cuda(), off, out, lse, ws)
    assert fs.fs_decode_status(ws) == 4
    compare(c, out, lse, qh, 4, 0.1, [(r, 0, r + 1) for r in (0, 50, 99)])
    c.close()
