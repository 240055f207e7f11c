"""fs_batch_tables against one request after the other: every written value, and everything else left as it was."""
import numpy as np
import pytest

import block_cache as plain
import paper_2509_06261_amd as fs

pytestmark = pytest.mark.gpu
MARK = -77


def make_pool(t, n_blocks=1 << 20):
    """A pool of n_blocks blocks that the calls only name (its memory is never touched)."""
    import torch
    block = fs.fs_block_bytes(fs.FS_KV_FP16, 1, 8, 1, t)
    mem = torch.empty(256, dtype=torch.uint8, device="cuda")
    pool = fs.fs_pool_create(block, n_blocks * block, mem)
    return pool, fs.fs_model_register_tokens(pool, fs.FS_KV_FP16, 1, 8, 1, t)[1], mem


def run(t, held, new, n_ids, max_blocks, n_tokens, seed=0, n_blocks=1 << 20, with_slots=True, with_held=True, spoil=0, offset=0):
    """offset: elements that every array begins behind an allocation's start (alignment); returns (got, want)."""
    import torch
    rng = np.random.default_rng(seed)
    held, new = np.asarray(held, np.int64), np.asarray(new, np.int64)
    n = len(new)
    ids = rng.permutation(max(n_ids, 1) * 2)[:n_ids].astype(np.int64)
    table = rng.integers(0, n_blocks, (n, max_blocks))
    if spoil:  # ids and held blocks that are none of the pool
        ids[rng.random(n_ids) < 0.2] = n_blocks + 5
        table[rng.random(table.shape) < 0.2] = -3

    def dev(x, dtype=torch.int32):
        x = np.asarray(x)
        buf = torch.full((x.size + offset + 8,), MARK, dtype=dtype, device="cuda")
        buf[offset:offset + x.size] = torch.from_numpy(np.ascontiguousarray(x.reshape(-1).astype(np.int64))).to("cuda", dtype)
        return buf, buf[offset:offset + x.size].view(x.shape)

    full = lambda k: np.full(k, MARK)  # noqa: E731
    bufs = dict(table=dev(table), seq_lens=dev(full(n)), q_offsets=dev(full(n + 1)), seq_idx=dev(full(n_tokens)), pos=dev(full(n_tokens)),
                slots=dev(full(n_tokens), torch.int64), status=dev(full(1)))
    held_d, new_d, ids_d = dev(held)[1], dev(new)[1], dev(ids)[1]
    pool, m, mem = make_pool(t, n_blocks)
    b = {k: v[1] for k, v in bufs.items()}
    fs.fs_batch_tables(pool, m, held_d if with_held else None, new_d, ids_d, b["table"], b["seq_lens"], b["q_offsets"], b["seq_idx"], b["pos"],
                       b["slots"] if with_slots else None, b["status"])
    torch.cuda.synchronize()
    fs.fs_pool_destroy(pool)
    for buf, _ in bufs.values():  # nothing outside the arrays
        x = buf.cpu().numpy()
        assert (x[:offset] == MARK).all() and (x[len(x) - 8:] == MARK).all()
    want = plain.tables(held, new, ids, table, t, n_tokens, n_blocks, with_held)
    if not with_slots:
        want["slots"] = full(n_tokens)
    return {k: v.cpu().numpy() for k, v in b.items()}, want


def check(got, want):
    for k, w in want.items():
        assert np.array_equal(got[k].reshape(-1), np.reshape(w, -1)), (k, got[k], w)


def lengths(n, lo, hi, seed):
    return np.random.default_rng(seed).integers(lo, hi + 1, n)


@pytest.mark.parametrize("t", [1, 7, 16, 127])
@pytest.mark.parametrize("n", [1, 2, 63, 1023, 1024, 1025, 2500])
def test_decode_steps(n, t):
    held = lengths(n, 0, 6 * t, n)
    check(*run(t, held, np.ones(n), n, 8, n, seed=t))


@pytest.mark.parametrize("t,n,hi,spare", [(31, 300, 900, 0), (16, 40, 5000, 77), (8, 1500, 60, 4096), (60, 3, 30000, 1), (128, 1, 200000, 0)])
@pytest.mark.parametrize("held_hi", [0, 3000])
def test_prompts_and_chunks(t, n, hi, spare, held_hi):
    held, new = lengths(n, 0, held_hi, 1), lengths(n, 0, hi, 2)
    blocks = int((-(-(held + new) // t) + -held // t).sum())
    check(*run(t, held, new, blocks + 5, -(-(hi + held_hi) // t) + 1, int(new.sum()) + spare, with_held=held_hi > 0))


@pytest.mark.parametrize("offset", [1, 3])
def test_unaligned_arrays_and_no_slots(offset):
    held, new = lengths(70, 0, 200, 3), lengths(70, 0, 150, 4)
    for with_slots in (True, False):
        check(*run(33, held, new, 2000, 12, int(new.sum()) + 9, offset=offset, with_slots=with_slots))


def test_nothing_new():
    check(*run(16, lengths(90, 0, 100, 5), np.zeros(90), 0, 9, 0))
    check(*run(16, lengths(90, 0, 100, 5), np.zeros(90), 3, 9, 5))  # five tokens of padding
    check(*run(16, np.zeros(1), np.zeros(1), 0, 1, 0))


def test_lists_that_are_too_short():
    held, new = lengths(200, 0, 100, 6), lengths(200, 0, 300, 7)
    total = int(new.sum())
    for n_ids, n_tokens in ((50, total), (5000, total // 2), (50, total // 3), (0, total), (5000, 1), (5000, 0)):
        got, want = run(16, held, new, n_ids, 40, n_tokens)
        check(got, want)
        assert got["status"][0] == 2
    # the cut is where a request begins, ends, and between requests of a later window
    new = np.full(3000, 5)
    for n_tokens in (5 * 1024, 5 * 1024 - 1, 5 * 2048 + 2):
        check(*run(4, np.zeros(3000), new, 6000, 3, n_tokens))


def test_lengths_out_of_range():
    held = np.array([5, -3, 1000, 20, 2 ** 31 - 1, -2 ** 31, 64])
    new = np.array([-1, 10, 5, 1000, 7, 2 ** 31 - 1, 0])
    got, want = run(16, held, new, 100, 4, 300)
    check(got, want)
    assert got["status"][0] == 1
    got, want = run(16, held, new, 3, 4, 30)
    check(got, want)
    assert got["status"][0] == 3


def test_blocks_outside_the_pool_have_no_slots():
    got, want = run(8, lengths(100, 0, 50, 8), lengths(100, 0, 50, 9), 1500, 14, 6000, n_blocks=1 << 12, spoil=1)
    check(got, want)
    assert (got["slots"] == -1).sum() > 6000 - want["q_offsets"][-1]


def test_slots_pass_32_bits():
    # 2^25 blocks of 2^17 tokens: rows of the pool beyond 2^40
    t, n_blocks = 1 << 17, 1 << 12
    got, want = run(t, [0, 3], [2, 2], 2, 1, 4, n_blocks=n_blocks)
    check(got, want)
    ids = [(1 << 31) - 5]
    table = plain.tables([0], [3], ids, np.array([[0]]), t, 3, 1 << 31)
    assert table["slots"].max() > 1 << 40  # (what the definition says; a pool of that many blocks cannot be had)


def test_captured_and_replayed():
    """A step whose lengths live on the device: a captured call, replayed on lengths that eager work changes in between."""
    import torch
    t, n, steps = 8, 50, 6
    pool, m, mem = make_pool(t)
    held = torch.randint(0, 30, (n,), dtype=torch.int32, device="cuda")
    new = torch.ones(n, dtype=torch.int32, device="cuda")
    ids = torch.arange(1000, 1000 + n, dtype=torch.int32, device="cuda")
    z = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    table, lens, off, seq, pos, slots, status = z(n, 12), z(n), z(n + 1), z(n + 10), z(n + 10), z(n + 10, dt=torch.int64), z(1)
    call = lambda: fs.fs_batch_tables(pool, m, held, new, ids, table, lens, off, seq, pos, slots, status)  # noqa: E731
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call()
    for k in range(steps):
        held.copy_(torch.randint(0, 60, (n,), dtype=torch.int32, device="cuda"))
        new.copy_(torch.randint(0, 2, (n,), dtype=torch.int32, device="cuda"))
        before = table.cpu().numpy().astype(np.int64)
        g.replay()
        torch.cuda.synchronize()
        want = plain.tables(held.cpu().numpy(), new.cpu().numpy(), np.arange(1000, 1000 + n), before, t, n + 10, 1 << 20)
        check(dict(table=table.cpu().numpy(), seq_lens=lens.cpu().numpy(), q_offsets=off.cpu().numpy(), seq_idx=seq.cpu().numpy(), pos=pos.cpu().numpy(),
                   slots=slots.cpu().numpy(), status=status.cpu().numpy()), want)
    fs.fs_pool_destroy(pool)
