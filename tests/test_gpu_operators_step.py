"""The operators in a row, as a serving loop uses them: block tables and maps, rotation and append, attention -- prompts first, then
steps, eager and captured, over an FP8_BLOCK cache; against the definitions in 64 bits."""
import math

import numpy as np
import pytest

import block_cache as plain
import paper_2509_06261_amd as fs

pytestmark = pytest.mark.gpu


class Server:
    def __init__(self, heads=2, group=4, d=128, t=24, r=96, seqs=5, longest=400, seed=0):
        import torch
        self.heads, self.group, self.d, self.t, self.seqs, self.r = heads, group, d, t, seqs, r
        self.rng = np.random.default_rng(seed)
        p = plain.layout(heads, d, t, 1)
        self.n = seqs * (-(-longest // t)) + 4
        self.mem = torch.zeros(self.n * p["block"], dtype=torch.uint8, device="cuda")
        self.pool = fs.fs_pool_create(p["block"], self.mem.numel(), self.mem)
        _, self.model = fs.fs_model_register_tokens(self.pool, fs.FS_KV_FP8_BLOCK, heads, d, 1, t)
        fs.fs_model_set_rope(self.pool, self.model, fs.make_rope(r, 10000.0))
        self.freq = plain.frequencies(r, 10000.0, "none")
        self.nb = -(-longest // t)
        z = lambda *s: torch.full(s, -1, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.lens, self.offsets = z(seqs, self.nb), torch.zeros(seqs, dtype=torch.int32, device="cuda"), z(seqs + 1)
        self.held = np.zeros(seqs, np.int64)
        self.cache = [plain.BlockCache(self.n, heads, t, d) for _ in range(2)]

    def maps(self, n):
        import torch
        return [torch.empty(n, dtype=dt, device="cuda") for dt in (torch.int32, torch.int32, torch.int64)]

    def blocks_for(self, new):
        need = -(-(self.held + new) // self.t) + -self.held // self.t  # ceil - ceil
        rc, ids = fs.fs_blocks_alloc(self.pool, self.model, int(need.sum()))
        assert rc == fs.FS_OK
        return ids

    def close(self):
        fs.fs_pool_destroy(self.pool)

    # the definitions: what the cache holds is taken from the pool, so that a rounding that falls the other way (the keys are
    # rotated in fp32) does not count again in what follows
    def take(self, seq, pos, k, v):
        rk, _ = plain.rotate(k, pos, self.freq, True)
        table = self.table.cpu().numpy()
        blk, slot = table[seq, pos // self.t], pos % self.t
        got = plain.views(self.mem, self.heads, self.d, self.t, 1, 0)
        for which, (w, x) in enumerate(zip(self.cache, (rk, v))):
            w.append(x, blk, slot)
            for b in np.unique(blk):
                assert (got[2][b, :, which].cpu().numpy() == 2.0 ** w.e[b]).all()
                codes = plain.e4m3_value(got[which][b, :, :w.used[b]].cpu().numpy())
                off = np.abs(codes - w.codes[b][:, :w.used[b]])
                # one step between neighbouring codes where fp32 and 64 bits round to different sides
                assert (off <= np.maximum(np.abs(codes) / 8, 2.0 ** -9) * 1.001).all() and (off > 0).mean() < 0.01
                w.codes[b][:, :w.used[b]] = codes

    def rows(self, i, n, table):
        at = np.arange(n)
        blk, slot = table[i, at // self.t], at % self.t
        return [w.codes[blk, :, slot] * 2.0 ** w.e[blk][:, :, None] for w in self.cache]

    def check(self, out, lse, q_out, rows):
        out, lse, q = (x.double().cpu().numpy() for x in (out, lse, q_out))
        table = self.table.cpu().numpy()
        for r, i, n in rows:
            k, v = self.rows(i, n, table)
            for h in range(self.heads):
                g = slice(h * self.group, (h + 1) * self.group)
                want, want_lse, s = plain.attention(q[r, g], k[:, h], v[:, h], 1 / math.sqrt(self.d))
                assert (np.abs(out[r, g] - want) <= plain.out_tolerance(want, s, n, np.abs(v[:, h]).max())).all(), (r, i, n)
                assert np.abs(lse[r, g] - want_lse).max() < 2e-5 + 2e-6 * np.abs(want_lse).max()


def new_rows(s, n):
    import torch
    width = (s.group + 2) * s.heads * s.d
    qkv = torch.from_numpy(s.rng.standard_normal((n, width)).astype(np.float16)).cuda()
    q, k, v = qkv.split([s.group * s.heads * s.d, s.heads * s.d, s.heads * s.d], dim=1)
    return [x.view(n, -1, s.d) for x in (q, k, v)]


def host(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("shape", [dict(), dict(heads=1, group=8, d=64, t=17, r=64), dict(heads=3, group=1, d=256, t=9, r=40, seqs=3, longest=120)])
def test_prompts_then_steps(shape):
    import torch
    s = Server(**shape)
    scale = 1 / math.sqrt(s.d)
    longest = s.nb * s.t
    prompts = s.rng.integers(1, longest // 2, s.seqs)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for new in (np.where(np.arange(s.seqs) % 2 == 0, prompts, 0), np.where(np.arange(s.seqs) % 2 == 1, prompts, 5)):  # a chunk behind some
            n = int(new.sum())
            ids = torch.from_numpy(s.blocks_for(new)).cuda()
            seq, pos, slots = s.maps(n + 7)
            status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
            new_d, held_d = (torch.from_numpy(x.astype(np.int32)).cuda() for x in (new, s.held))
            fs.fs_batch_tables(s.pool, s.model, held_d, new_d, ids, s.table, s.lens, s.offsets, seq, pos, slots, status)
            q, k, v = new_rows(s, n + 7)  # (seven tokens of padding)
            q_out = torch.full(q.shape, 3.0, dtype=torch.float16, device="cuda")
            fs.fs_rope_append(s.pool, s.model, 0, q, k, v, seq, pos, s.table, q_out)
            off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
            out, lse = torch.empty_like(q_out[:n]), torch.empty((n, q.shape[1]), device="cuda")
            ws = torch.empty(fs.fs_prefill_workspace_bytes(s.seqs), dtype=torch.uint8, device="cuda")
            rows = slice(0, n)
            # (a request without a length takes no part in the attention call yet)
            live = np.flatnonzero(s.held + new)
            index = torch.from_numpy(live).cuda()
            off_live = np.concatenate([off[live], off[-1:]]).astype(np.int32)
            fs.fs_prefill_attention(s.pool, s.model, 0, q.shape[1], scale, q_out[rows], s.table[index].contiguous(), s.lens[index].contiguous(),
                                    torch.from_numpy(off_live).cuda(), off_live, out, lse, ws)
            assert fs.fs_decode_status(ws) == 0 and int(status) == 0
            assert (q_out[n:] == 3).all() and (seq[n:] == -1).all()
            sh, ph = seq[:n].cpu().numpy(), pos[:n].cpu().numpy()
            s.take(sh, ph, host(k[:n]), host(v[:n]))
            s.held = s.held + new
            assert np.array_equal(s.lens.cpu().numpy(), s.held)
            pick = s.rng.choice(n, min(n, 30), replace=False)
            s.check(out, lse, q_out, [(int(r), int(sh[r]), int(ph[r]) + 1) for r in pick])
    # steps: lengths on the device only; the same calls captured once and replayed between eager ones
    one = torch.ones(s.seqs, dtype=torch.int32, device="cuda")
    held_d = s.lens.clone()
    ids = torch.zeros(s.seqs, dtype=torch.int32, device="cuda")
    seq, pos, slots = s.maps(s.seqs)
    q, k, v = new_rows(s, s.seqs)
    q_out = torch.empty(q.shape, dtype=torch.float16, device="cuda")
    out, lse = torch.empty_like(q_out), torch.empty(q.shape[:2], device="cuda")
    batch = fs.make_batch(s.model, 0, q.shape[1], scale, q_out, s.table, s.lens, out, lse)
    ws = torch.empty(fs.fs_decode_workspace_bytes(s.pool, [batch]), dtype=torch.uint8, device="cuda")

    def step():
        fs.fs_batch_tables(s.pool, s.model, held_d, one, ids, s.table, s.lens, s.offsets, seq, pos, slots)
        fs.fs_rope_append(s.pool, s.model, 0, q, k, v, seq, pos, s.table, q_out)
        fs.fs_decode_attention(s.pool, s.model, 0, q.shape[1], scale, q_out, s.table, s.lens, out, lse, ws)
        held_d.copy_(s.lens)

    graph = None
    for k_step in range(12):
        fresh = s.blocks_for(np.ones(s.seqs, np.int64))
        ids[:len(fresh)] = torch.from_numpy(fresh).cuda()
        qkv = new_rows(s, s.seqs)
        for a, b in zip((q, k, v), qkv):
            a.copy_(b * (1.0 + k_step))  # rows that grow, and with them the scales
        if k_step < 4 or k_step % 4 == 3:
            step()
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step()
            graph.replay()
        torch.cuda.synchronize()
        assert fs.fs_decode_status(ws) == 0
        s.take(np.arange(s.seqs), s.held, host(k), host(v))
        assert np.array_equal(pos.cpu().numpy(), s.held)
        s.held = s.held + 1
        s.check(out, lse, q_out, [(i, i, int(s.held[i])) for i in range(s.seqs)])
    s.close()


def test_calls_follow_the_current_stream():
    """Behind a kernel that keeps a stream busy the calls see what that stream brings before them."""
    import torch
    s = Server(seqs=2, longest=60)
    q, k, v = new_rows(s, 2)
    held, one = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    ids = torch.from_numpy(s.blocks_for(np.ones(2, np.int64))).cuda()
    seq, pos, slots = s.maps(2)
    late, q_out, back = torch.zeros_like(q), torch.zeros((2, 8, 128), dtype=torch.float16, device="cuda"), torch.zeros((2, 8, 128), dtype=torch.float16, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)
        late.copy_(q)
        held.fill_(7)
        fs.fs_batch_tables(s.pool, s.model, held, one, ids, s.table, s.lens, s.offsets, seq, pos, slots)
        fs.fs_rope_append(s.pool, s.model, 0, late.contiguous(), k, v, seq, pos, s.table, q_out)
        fs.fs_rope(s.pool, s.model, q_out, pos, back, inverse=True)
    stream.synchronize()
    assert pos.tolist() == [7, 7]
    # there and back: two roundings to fp16
    torch.testing.assert_close(back, q, rtol=0, atol=2 * 2.0 ** -11 * 6)
    s.close()
