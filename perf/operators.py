"""The operators around a KV slab pool that a decoder layer calls between its projections, timed call by call.

Three belong together and are measured alone and in a row:

* block tables and token maps from the requests' lengths (``fs_batch_tables``),
* rotary positions, by themselves (``fs_rope``) and on the way into the cache (``fs_rope_append``: queries and keys are
  rotated, keys and values stored),
* attention over a cache of E4M3 codes with one power-of-two scale for each (block, KV head, K or V)
  (``FS_KV_FP8_BLOCK``), for single tokens and for prompts and chunks.

A case's ``t`` is the tokens of a block; a block is one slab, laid out as the library documents it: layers one after the
other, in a layer the KV heads' K and V rows, and (FP8_BLOCK) behind them the K and V scale of every head.  The plain
forms read and write the same bytes through strided views.  Two layers lie in a block; the second one is used.
"""
import math

import numpy as np
import torch

own = False  # whether run() calls the framework's operators (or computes the plain forms)

_LAYERS, _LAYER = 2, 1
_E_MIN, _E_MAX = -15, 7  # exponents of a block's scale


def listed():
    return [
        # one new token for each of a few chats, what a captured decode step of a small server asks for: latency only
        _tables("tables-decode-few", 8, 1, 256, 1, 1, 16),
        # a step's admission: thousands of prompts, lengths from one token on, blocks of an odd size; bound by writing the maps
        _tables("tables-prompts-many", 2048, 0, 0, 1, 900, 31, spare=1000),
        # queries of a batch of prompts, taken out of a fused projection's rows
        _rope("rope-queries", 16384, 32, 128, 128, "halves", "none", 4096, "fp16", wide=6144),
        # rows of an odd count, part of the head in neighbouring pairs, fp32, positions far behind the trained ones; the way back
        _rope("rope-far-partial", 1999, 5, 64, 32, "pairs", "wavelength", 900000, "fp32", inverse=True),
        # a decode step's newest tokens into an FP16 cache
        _append("rope-append-decode-fp16", "fp16", 64, 1, 1, 512, 4096, 8, 4, 128, 16, 128, "halves", "wavelength"),
        # prompts of a batch into the cache with block scales, rows of a fused projection
        _append("rope-append-prompts", "fp8", 32, 100, 4000, 0, 0, 8, 4, 128, 63, 128, "halves", "dimension", wide=True),
        # the ordinary decode call: 64 chats, four query heads to a KV head
        _decode("decode-chats", 64, 512, 4096, 8, 4, 128, 64),
        # a few long documents, eight query heads to a KV head; the lengths are known on the device only
        _decode("decode-long-few", 5, 9000, 32768, 8, 8, 128, 126, lens_known=False),
        # the largest: a batch of many chats
        _decode("decode-many", 256, 1024, 8192, 8, 4, 128, 127),
        # chunked prefill: 512 new tokens of a few requests behind long contexts
        _prefill("prefill-chunk", 4, 3000, 16384, 512, 8, 4, 128, 64),
        # whole prompts of a small model
        _prefill("prefill-prompts-d64", 12, 200, 2000, 0, 8, 4, 64, 50),
        # a whole step of one layer, lengths on the device: tables and maps, rotation and append, attention
        _step("step-chats", 128, 200, 3000, 8, 4, 128, 63, 128, "halves", "none"),
    ]


def _tables(name, seqs, held_lo, held_hi, new_lo, new_hi, t, spare=0):
    return dict(name=name, kind="tables", seqs=seqs, held_lo=held_lo, held_hi=held_hi, new_lo=new_lo, new_hi=new_hi, t=t, spare=spare)


def _rope(name, tokens, heads, d, rotary, layout, scaling, far, src, wide=0, inverse=False):
    return dict(name=name, kind="rope", tokens=tokens, heads=heads, d=d, rotary=rotary, layout=layout, scaling=scaling, far=far,
                src=src, wide=wide, inverse=inverse)


def _append(name, fmt, seqs, new_lo, new_hi, held_lo, held_hi, h, g, d, t, rotary, layout, scaling, src="fp16", wide=False):
    return dict(name=name, kind="append", fmt=fmt, seqs=seqs, new_lo=new_lo, new_hi=new_hi, held_lo=held_lo, held_hi=held_hi, h=h,
                g=g, d=d, t=t, rotary=rotary, layout=layout, scaling=scaling, src=src, wide=wide)


def _decode(name, seqs, lo, hi, h, g, d, t, lens_known=True):
    return dict(name=name, kind="decode", fmt="fp8", seqs=seqs, lo=lo, hi=hi, h=h, g=g, d=d, t=t, lens_known=lens_known)


def _prefill(name, seqs, lo, hi, chunk, h, g, d, t):
    return dict(name=name, kind="prefill", fmt="fp8", seqs=seqs, lo=lo, hi=hi, chunk=chunk, h=h, g=g, d=d, t=t)


def _step(name, seqs, lo, hi, h, g, d, t, rotary, layout, scaling):
    return dict(name=name, kind="step", fmt="fp8", seqs=seqs, held_lo=lo, held_hi=hi, new_lo=1, new_hi=1, h=h, g=g, d=d, t=t,
                rotary=rotary, layout=layout, scaling=scaling, src="fp16", wide=True)


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))))

    kind = rng.choices(["tables", "rope", "append", "decode", "prefill", "step"], [0.14, 0.16, 0.22, 0.22, 0.16, 0.1])[0]
    h, g, d = rng.choice([(8, 4, 128), (8, 8, 128), (4, 2, 128), (40, 1, 128), (8, 4, 64), (4, 1, 64), (4, 4, 256), (2, 16, 128)])
    t = rng.choice([8, 9, 16, 31, 32, 60, 64, 127, 128, rng.randint(8, 200)])
    rotary = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
    layout, scaling = rng.choice(["halves", "pairs"]), rng.choice(["none", "linear", "base", "wavelength", "dimension"])
    if scaling == "base":
        rotary = max(rotary, 4)
    src = rng.choice(["fp16", "fp16", "fp32"])
    if kind == "tables":
        held = rng.choice([0, log_int(1, 20000)])
        new = rng.choice([1, log_int(1, 2000)])
        c = _tables("", log_int(1, min(3000, 900000 // new, 500000 * t // (held + new))), min(1, held), held, rng.choice([0, 1]) if new > 1 else 1, new, t, rng.choice([0, log_int(1, 3000)]))
    elif kind == "rope":
        heads = rng.choice([1, 2, 5, 8, 32, 40])
        c = _rope("", log_int(1, min(60000, 67e6 / (heads * d))), heads, d, rotary, layout, scaling, log_int(100, 2000000), src,
                  rng.choice([0, heads * d + 8 * rng.randint(1, 500)]), rng.random() < 0.3)
    elif kind == "append":
        hi = rng.choice([1, 1, log_int(2, 4000)])
        held = rng.choice([0, log_int(1, 8000)])
        # (a cache as large as the tokens held; what is new is bounded by the widest rows)
        most = min(256, 65000 * 1024 / (h * d) / hi, 600000 * 1024 / (h * d) / (held + hi))
        c = _append("", rng.choice(["fp16", "fp8", "fp8"]), log_int(1, max(1, most)), rng.randint(1, hi), hi, min(1, held), held, h,
                    g, d, t, rotary, layout, scaling, src, rng.random() < 0.5)
    elif kind == "prefill":
        hi = log_int(16, 6000)
        chunk = rng.choice([0, 0, log_int(1, 1024)])
        rows = min(chunk, hi) if chunk else hi
        most = min(48, 1.4e8 / (h * g * rows * hi / 8), 60000 / hi)
        c = _prefill("", log_int(1, max(1, most)), rng.randint(1, hi), hi, chunk, h, g, d, t)
    else:
        hi = log_int(1, 16384 if kind == "decode" else 4000)
        most = min(256, (1.9e9 if kind == "decode" else 0.5e9) / (hi * 2 * h * d))
        seqs = log_int(1, max(1, most))
        if kind == "decode":
            c = _decode("", seqs, rng.randint(1, hi), hi, h, g, d, t, rng.random() < 0.6)
        else:
            c = _step("", seqs, rng.randint(1, hi), hi, h, g, d, t, rotary, layout, scaling)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ a case's arithmetic
def _spread(n, lo, hi):
    """n lengths: evenly spaced quantiles of lo .. hi, the same for every seed (the seed orders them)."""
    u = (np.arange(n) + 0.5) / n
    return np.clip(np.floor(lo + u * (hi - lo + 1)), lo, hi).astype(np.int64)


def _lens(case):
    """(held, new) tokens of every sequence before its seed's order."""
    n = case["seqs"]
    if case["kind"] in ("decode", "prefill"):
        total = _spread(n, case["lo"], case["hi"])
        new = np.ones_like(total) if case["kind"] == "decode" else np.minimum(total, case["chunk"]) if case["chunk"] else total
        return total - new, new
    return _spread(n, case["held_lo"], case["held_hi"])[::-1].copy(), _spread(n, case["new_lo"], case["new_hi"])


def _seeded_lens(case, seed):
    held, new = _lens(case)
    order = np.random.default_rng([seed, 1]).permutation(len(held))
    return held[order], new[order]


def _layout(case):
    """Bytes of the pieces of a block."""
    row = case["d"] * (2 if case["fmt"] == "fp16" else 1)
    tile = -(-case["t"] * row // 16) * 16
    chunk = 2 * tile
    scales = case["h"] * chunk
    layer = -(-(scales + (8 * case["h"] if case["fmt"] == "fp8" else 0)) // 256) * 256
    return dict(row=row, tile=tile, chunk=chunk, scales=scales, layer=layer, block=_LAYERS * layer)


def _row_bytes(case):
    """Bytes of K and V of a token, all heads of one layer (with its share of the block's scales)."""
    return 2 * case["h"] * (2 * case["d"] if case["fmt"] == "fp16" else case["d"] + 4 / case["t"])


def work(case):
    kind, nbytes, flops = case["kind"], 0.0, 0.0
    if kind == "rope":
        el = 4 if case["src"] == "fp32" else 2
        n = case["tokens"] * case["heads"]
        return {"bytes": n * case["d"] * 2.0 * el + 4 * case["tokens"], "flops": 3.0 * n * case["rotary"]}
    held, new = _lens(case)
    n, t = float(new.sum()), case["t"]
    if kind in ("tables", "step"):
        blocks = float((-(-(held + new) // t) - -(-held // t)).sum())
        nbytes += 16 * len(held) + 8 * blocks + 16 * (n + case.get("spare", 0))
    if kind in ("append", "step"):
        h, g, d = case["h"], case["g"], case["d"]
        el = 4 if case["src"] == "fp32" else 2
        nbytes += n * ((g + 2) * h * d * el + g * h * d * 2 + _row_bytes(case) + 8)
        flops += 3.0 * n * (g + 1) * h * case["rotary"]
    if kind in ("decode", "prefill", "step"):
        h, g, d = case["h"], case["g"], case["d"]
        nbytes += float((held + new).sum()) * _row_bytes(case) + n * h * g * (4 * d + 4)
        flops += 4.0 * d * h * g * float((new * held + new * (new + 1) // 2).sum())
    return {"bytes": nbytes, "flops": flops}


_BASE, _ORIGINAL = 500000.0, 8192


def _scaling(case):
    """(factor, low, high, amplitude) of the case's way to far positions."""
    return {"none": (1.0, 0.0, 0.0, 1.0), "linear": (4.0, 0.0, 0.0, 1.0), "base": (8.0, 0.0, 0.0, 1.0),
            "wavelength": (8.0, 1.0, 4.0, 1.0), "dimension": (16.0, 1.0, 32.0, 0.1 * math.log(16.0) + 1.0)}[case["scaling"]]


def _frequencies(case):
    """Radians per position of every pair."""
    r, (factor, low, high, _) = case["rotary"], _scaling(case)
    i = np.arange(r // 2, dtype=np.float64)
    base = _BASE * factor ** (r / (r - 2)) if case["scaling"] == "base" else _BASE
    f = base ** (-2 * i / r)
    if case["scaling"] == "linear":
        return f / factor
    if case["scaling"] == "wavelength":  # pairs that turn often within the original positions keep their frequency
        keep = np.clip((_ORIGINAL * f / (2 * math.pi) - low) / (high - low), 0, 1)
        return f * (keep + (1 - keep) / factor)
    if case["scaling"] == "dimension":  # the same, linear in the pair's index
        at = [r * math.log(_ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(_BASE)) for turns in (high, low)]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        stretch = np.clip((i - first) / max(last - first, 0.001), 0, 1)
        return f * (1 - stretch) + f / factor * stretch
    return f


# ------------------------------------------------------------------------------------------------------------- inputs
def _gen(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(np.random.SeedSequence(key).generate_state(1, np.uint64)[0] >> 1))
    return g


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def _dtype(case):
    return torch.float32 if case["src"] == "fp32" else torch.float16


def _views(case, mem):
    """K rows, V rows [block][head][token][bytes] and scales [block][head][K, V] of the layer in use."""
    p, n = _layout(case), mem.numel() // _layout(case)["block"]
    at = _LAYER * p["layer"]
    size, step = (n, case["h"], case["t"], p["row"]), (p["block"], p["chunk"], p["row"], 1)
    k, v = (mem.as_strided(size, step, at + which * p["tile"]) for which in (0, 1))
    if case["fmt"] == "fp16":
        return k, v, None
    return k, v, mem.view(torch.float32).as_strided((n, case["h"], 2), (p["block"] // 4, 2, 1), (at + p["scales"]) // 4)


def _fill(case, mem, seed):
    """Every block filled: N(0, 1) rows of heads and blocks that differ in size, as an append of whole blocks stores them."""
    k, v, scales = _views(case, mem)
    g = _gen(seed, 2)
    some = max(1, (1 << 26) // (case["h"] * case["t"] * case["d"]))
    for at in range(0, k.shape[0], some):
        for which, rows in enumerate((k, v)):
            part = rows[at:at + some]
            if scales is None:
                part.view(torch.float16).copy_(torch.randn(part.shape[:-1] + (case["d"],), generator=g, device="cuda", dtype=torch.float16))
                continue
            x = torch.randn(part.shape, generator=g, device="cuda", dtype=torch.float16).float()
            x *= torch.exp(0.5 * torch.randn(part.shape[:2] + (1, 1), generator=g, device="cuda"))
            e = _exponent(x.abs().amax((2, 3)))
            part.copy_(_codes(x, e[:, :, None, None]).view(torch.uint8))
            scales[at:at + some, :, which] = torch.exp2(e)


class _State:
    """What a serving program holds before the call."""
    pool = None

    def __del__(self):
        if self.pool is not None:
            import paper_2509_06261_amd as fs
            fs.fs_pool_destroy(self.pool)


def _tokens(held, new):
    """(sequence, position) of the new tokens, sequence by sequence."""
    start = np.cumsum(new) - new
    return np.repeat(np.arange(len(new)), new), np.arange(int(new.sum())) - np.repeat(start, new) + np.repeat(held, new)


def prepare(case, seed):
    s = _State()
    s.case, kind = case, case["kind"]
    rng = np.random.default_rng([seed, 3])
    if "rotary" in case:
        s.freq, s.amplitude = torch.from_numpy(_frequencies(case)).cuda(), _scaling(case)[3]
    if kind == "rope":
        n, w = case["tokens"], case["heads"] * case["d"]
        x = torch.randn((n, case["wide"] or w), generator=_gen(seed, 4), device="cuda", dtype=_dtype(case))
        s.x = x[:, :w].view(n, case["heads"], case["d"])
        s.pos = _i32(rng.integers(0, case["far"], n))
        s.out = torch.empty_like(s.x, memory_format=torch.contiguous_format)
        s.model_shape = ("fp16", 1, case["d"], 16)
    else:
        held, new = _seeded_lens(case, seed)
        t, total = case["t"], held + new
        blocks, old = -(-total // t), -(-held // t)
        s.blocks = n_blocks = int(blocks.sum()) + case.get("spare", 0) // 8 + 1
        ids = rng.permutation(n_blocks)  # a pool that has been in use hands its blocks out in any order
        table = np.full((len(new), int(max(blocks.max(), 1)) + 1), -1)
        fresh, at = [], 0
        for i in range(len(new)):
            table[i, :blocks[i]] = ids[at:at + blocks[i]]
            fresh.append(table[i, old[i]:blocks[i]].copy())
            if kind in ("tables", "step"):
                table[i, old[i]:] = -1
            at += blocks[i]
        s.table, s.held, s.new = _i32(table), _i32(held), _i32(new)
        s.ids = _i32(np.concatenate(fresh + [ids[at:]]))
        seq, pos = _tokens(held, new)
        n = len(seq)
        s.seq, s.pos = _i32(seq), _i32(pos)
        s.offsets_host = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        s.offsets, s.lens, s.lens_host = _i32(s.offsets_host), _i32(total), total.astype(np.int32)
        if kind == "tables":
            s.model_shape = ("fp16", 1, 8, t)
            s.capacity = n + case["spare"]
        else:
            s.model_shape = (case["fmt"], case["h"], case["d"], t)
            s.capacity = n
            s.mem = torch.zeros(n_blocks * _layout(case)["block"], dtype=torch.uint8, device="cuda")
            if kind != "append" or case["held_hi"]:
                _fill(case, s.mem, seed)
            h, g, d = case["h"], case["g"], case["d"]
            s.scale = 1.0 / math.sqrt(d)
            gen = _gen(seed, 5)
            if kind in ("append", "step"):
                width = (g + 2) * h * d
                qkv = torch.randn((n, width), generator=gen, device="cuda", dtype=_dtype(case))
                parts = qkv.split([g * h * d, h * d, h * d], dim=1)  # views of the fused projection's rows
                s.q, s.k, s.v = ((x if case["wide"] else x.contiguous()).view(n, -1, d) for x in parts)
            else:
                q = torch.randn((n, h * g, d), generator=gen, device="cuda", dtype=torch.float16)
                s.q = q * torch.linspace(0.5, 3.0, h * g, device="cuda", dtype=torch.float16).view(1, -1, 1)
            s.q_out = torch.empty((n, h * g, d), dtype=torch.float16, device="cuda")
            s.out = torch.empty((n, h * g, d), dtype=torch.float16, device="cuda")
            s.lse = torch.empty((n, h * g), dtype=torch.float32, device="cuda")
        if kind in ("tables", "step"):
            s.maps = dict(seq_lens=torch.empty_like(s.lens), q_offsets=torch.empty_like(s.offsets), **{
                k: torch.empty(s.capacity, dtype=torch.int64 if k == "slots" else torch.int32, device="cuda") for k in ("seq_idx", "pos", "slots")})
    if own:
        _hold(s)
    torch.cuda.synchronize()
    return s


def _hold(s):
    """The pool and the model that a program registers once, the rotation it sets, and workspaces."""
    import paper_2509_06261_amd as fs
    case = s.case
    fmt, h, d, t = s.model_shape
    fmt = {"fp16": fs.FS_KV_FP16, "fp8": fs.FS_KV_FP8_BLOCK}[fmt]
    block = fs.fs_block_bytes(fmt, h, d, _LAYERS, t)
    if case["kind"] in ("rope", "tables"):  # (the calls name the pool and its model, but touch no block)
        n = s.blocks if case["kind"] == "tables" else 1
        s.mem = torch.empty(n * block, dtype=torch.uint8, device="cuda")
    else:
        assert block == _layout(case)["block"]
        n = s.mem.numel() // block
    s.pool = fs.fs_pool_create(block, n * block, s.mem)
    _, s.model = fs.fs_model_register_tokens(s.pool, fmt, h, d, _LAYERS, t)
    rc, _ = fs.fs_blocks_alloc(s.pool, s.model, n)
    assert rc == fs.FS_OK
    if "rotary" in case:
        factor, low, high, amplitude = _scaling(case)
        kinds = {"none": fs.FS_ROPE_UNSCALED, "linear": fs.FS_ROPE_LINEAR, "base": fs.FS_ROPE_BASE,
                 "wavelength": fs.FS_ROPE_WAVELENGTH, "dimension": fs.FS_ROPE_DIMENSION}
        fs.fs_model_set_rope(s.pool, s.model, fs.make_rope(
            case["rotary"], _BASE, layout=fs.FS_ROPE_HALVES if case["layout"] == "halves" else fs.FS_ROPE_PAIRS, scaling=kinds[case["scaling"]],
            factor=factor, low=low, high=high, original_positions=_ORIGINAL, amplitude=amplitude))
    if case["kind"] in ("decode", "step"):
        s.batch = fs.make_batch(s.model, _LAYER, case["h"] * case["g"], s.scale, s.q if case["kind"] == "decode" else s.q_out, s.table, s.lens, s.out, s.lse,
                                s.lens_host if case.get("lens_known") else None)
        s.ws = torch.empty(fs.fs_decode_workspace_bytes(s.pool, [s.batch]), dtype=torch.uint8, device="cuda")
    if case["kind"] == "prefill":
        s.ws = torch.empty(fs.fs_prefill_workspace_bytes(case["seqs"]), dtype=torch.uint8, device="cuda")


# ----------------------------------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _cache(s):
    """The layer's cache as it is stored: rows in the cache's own type, and the scales they are multiplied by."""
    k, v, scales = _views(s.case, s.mem)
    if scales is None:
        return dict(k=k.view(torch.float16), v=v.view(torch.float16))
    return dict(k=k.view(torch.float8_e4m3fn), v=v.view(torch.float8_e4m3fn), scales=scales)


def _run_own(s):
    import paper_2509_06261_amd as fs
    case, kind = s.case, s.case["kind"]
    if kind == "rope":
        fs.fs_rope(s.pool, s.model, s.x, s.pos, s.out, inverse=case["inverse"])
        return s.out
    seq, pos = s.seq, s.pos
    if kind in ("tables", "step"):
        m = s.maps
        fs.fs_batch_tables(s.pool, s.model, s.held, s.new, s.ids, s.table, m["seq_lens"], m["q_offsets"], m["seq_idx"], m["pos"], m["slots"])
        if kind == "tables":
            return dict(m, table=s.table)
        seq, pos = m["seq_idx"], m["pos"]
    if kind in ("append", "step"):
        fs.fs_rope_append(s.pool, s.model, _LAYER, s.q, s.k, s.v, seq, pos, s.table, s.q_out)
        if kind == "append":
            return dict(_cache(s), q=s.q_out)
    n_q = case["h"] * case["g"]
    if kind == "step":
        fs.fs_decode_attention(s.pool, s.model, _LAYER, n_q, s.scale, s.q_out, s.table, m["seq_lens"], s.out, s.lse, s.ws)
        return dict(_cache(s), **m, table=s.table, q=s.q_out, out=s.out, lse=s.lse)
    if kind == "prefill":
        fs.fs_prefill_attention(s.pool, s.model, _LAYER, n_q, s.scale, s.q, s.table, s.lens, s.offsets, s.offsets_host, s.out, s.lse, s.ws)
    elif case["lens_known"]:
        fs.fs_decode_attention_multi(s.pool, [s.batch], s.ws)
    else:
        fs.fs_decode_attention(s.pool, s.model, _LAYER, n_q, s.scale, s.q, s.table, s.lens, s.out, s.lse, s.ws)
    return dict(out=s.out, lse=s.lse)


def _run_plain(s):
    kind = s.case["kind"]
    if kind == "rope":
        return _rotate(s, s.x.float(), s.pos, s.case["inverse"]).to(s.x.dtype)
    table, seq, pos, lens = s.table, s.seq, s.pos, s.lens
    if kind in ("tables", "step"):
        m = _plain_tables(s)
        if kind == "tables":
            return m
        table, seq, pos, lens = m["table"], m["seq_idx"], m["pos"], m["seq_lens"]
    if kind in ("append", "step"):
        q = _rotate(s, s.q.float(), pos).half()
        _store(s, _rotate(s, s.k.float(), pos), s.v.float(), table[seq.long(), (pos // s.case["t"]).long()].long(), (pos % s.case["t"]).long())
        if kind == "append":
            return dict(_cache(s), q=q)
        out, lse = _attend(s, q, table, lens, None)
        return dict(_cache(s), **m, q=q, out=out, lse=lse)
    out, lse = _attend(s, s.q, table, lens, s.offsets if kind == "prefill" else None)
    return dict(out=out, lse=lse)


def _plain_tables(s):
    t, n_seq, dev = s.case["t"], s.new.numel(), s.new.device
    held, new = s.held.long(), s.new.long()
    lens = held + new
    ends = new.cumsum(0)
    old = (held + t - 1) // t
    need = (lens + t - 1) // t - old
    last = need.cumsum(0)
    # the new blocks' places, in one list; a block id that nobody needs goes to a spare place at the end
    e = torch.arange(s.ids.numel(), device=dev)
    owner = torch.searchsorted(last, e, right=True)
    whose = owner.clamp(max=n_seq - 1)
    place = whose * s.table.shape[1] + old[whose] + e - (last - need)[whose]
    flat = torch.cat([s.table.view(-1), s.table.new_zeros(1)])
    flat[torch.where(owner < n_seq, place, flat.numel() - 1)] = s.ids
    table = flat[:-1].view_as(s.table)
    # the tokens
    i = torch.arange(s.capacity, device=dev)
    seq = torch.searchsorted(ends, i, right=True)
    live = seq < n_seq
    whose = seq.clamp(max=n_seq - 1)
    pos = held[whose] + i - (ends - new)[whose]
    slots = table[whose, torch.where(live, pos, 0) // t].long() * t + pos % t
    zero = torch.zeros(1, dtype=torch.int32, device=dev)
    return dict(table=table, seq_lens=lens.int(), q_offsets=torch.cat([zero, ends.int()]), seq_idx=torch.where(live, seq, -1).int(),
                pos=torch.where(live, pos, -1).int(), slots=torch.where(live, slots, -1))


def _rotate(s, x, pos, inverse=False):
    """x [token][head][d] in 32 bits, its first elements turned by position times frequency (angles in 64 bits)."""
    r = s.case["rotary"]
    angle = pos.double()[:, None] * s.freq[None]
    cos, sin = (angle.cos() * s.amplitude).float()[:, None], (angle.sin() * s.amplitude).float()[:, None]
    if inverse:
        sin = -sin
    y = x.clone()
    if s.case["layout"] == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * cos - b * sin, b * cos + a * sin
    return y


def _exponent(amax):
    """The least exponent e with amax <= 448 * 2^e, within the format's range."""
    mant, exp = torch.frexp(amax)
    e = torch.where(mant <= 0.875, exp - 9, exp - 8)
    return torch.where(amax > 0, e, _E_MIN).clamp(_E_MIN, _E_MAX).float()


def _codes(x, e):
    return (x * torch.exp2(-e)).clamp(-448, 448).to(torch.float8_e4m3fn)


def _store(s, k, v, blk, slot):
    """New rows [token][head][d] into the cache's bytes."""
    bytes_k, bytes_v, scales = _views(s.case, s.mem)
    if scales is None:
        bytes_k.view(torch.float16)[blk, :, slot] = k.half()
        bytes_v.view(torch.float16)[blk, :, slot] = v.half()
        return
    n = bytes_k.shape[0]
    first = torch.full((n,), s.case["t"], device=k.device).index_reduce_(0, blk, slot, "amin")  # lowest new slot of a block
    for which, (x, rows) in enumerate(((k, bytes_k), (v, bytes_v))):
        amax = torch.zeros((n, s.case["h"]), device=k.device).index_reduce_(0, blk, x.abs().amax(-1), "amax")
        # a block that begins anew forgets its scale; otherwise the scale only grows, and what is stored follows it
        before = torch.where((first == 0)[:, None], float(_E_MIN), scales[:, :, which].log2())
        touched = (first < s.case["t"])[:, None]
        after = torch.where(touched, torch.maximum(before, _exponent(amax)), before)
        grown = torch.nonzero(((after > before) & (first > 0)[:, None]).any(1))[:, 0]
        old = rows[grown].view(torch.float8_e4m3fn).float() * torch.exp2(before - after)[grown][:, :, None, None]
        rows[grown] = old.to(torch.float8_e4m3fn).view(torch.uint8)
        scales[:, :, which] = torch.where(touched, torch.exp2(after), scales[:, :, which])
        rows[blk, :, slot] = _codes(x, after[blk][:, :, None]).view(torch.uint8)


def _attend(s, q, table, lens, offsets):
    """Softmax attention over the cached tokens, all sequences padded to the longest; (out, lse)."""
    case = s.case
    h, g, d, t = (case[k] for k in "hgdt")
    n, longest = lens.numel(), int(s.lens_host.max())
    bytes_k, bytes_v, scales = _views(case, s.mem)
    at = torch.arange(longest, device=q.device)
    live = at[None] < lens[:, None]
    blk = torch.where(live, table[:, at // t], 0).long()
    k, v = (rows[blk, :, at % t].view(torch.float8_e4m3fn).float() * scales[blk, :, which, None] for which, rows in enumerate((bytes_k, bytes_v)))
    v = torch.where(live[:, :, None, None], v, 0.0).transpose(1, 2).contiguous()  # [sequence][head][token][d]
    k = torch.where(live[:, :, None, None], k, 0.0).permute(0, 2, 3, 1).contiguous()
    if offsets is None:
        rows, longest_new, of = q, 1, None
        seen = lens[:, None]
    else:
        new = (offsets[1:] - offsets[:-1]).long()
        longest_new = int((s.offsets_host[1:] - s.offsets_host[:-1]).max())
        r = torch.arange(longest_new, device=q.device)
        of = (offsets[:-1, None] + r).clamp(max=q.shape[0] - 1).long()
        rows = q[of]
        seen = lens[:, None] - new[:, None] + r + 1  # tokens that row r attends to
    x = rows.float().view(n, longest_new, h, g, d).permute(0, 2, 1, 3, 4).reshape(n, h, longest_new * g, d) * s.scale
    x = torch.matmul(x, k).view(n, h, longest_new, g, longest)
    x = x.masked_fill(at >= seen[:, None, :, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - top)
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.view(n, h, longest_new * g, longest), v).view(n, h, longest_new, g, d) / total
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(n, longest_new, h * g)
    out = out.permute(0, 2, 1, 3, 4).reshape(n, longest_new, h * g, d).half()
    if offsets is None:
        return out[:, 0], lse[:, 0]
    return out[s.seq.long(), s.pos.long() - (lens - new)[s.seq.long()]], lse[s.seq.long(), s.pos.long() - (lens - new)[s.seq.long()]]


# -------------------------------------------------------------------------------------------------- 64-bit definition
def _exact_rotation(case, x, pos, inverse=False):
    """Complex products in 64 bits."""
    r = case["rotary"]
    turn = torch.exp(1j * pos.double()[:, None, None] * torch.from_numpy(_frequencies(case)).cuda()) * _scaling(case)[3]
    x = x.double()
    head = x[..., :r].reshape(x.shape[:-1] + ((2, r // 2) if case["layout"] == "halves" else (r // 2, 2)))
    if case["layout"] == "halves":
        head = head.transpose(-1, -2)
    z = torch.complex(head[..., 0].contiguous(), head[..., 1].contiguous()) * (turn.conj() if inverse else turn)
    z = torch.stack([z.real, z.imag], -2 if case["layout"] == "halves" else -1).reshape(x.shape[:-1] + (r,))
    return torch.cat([z, x[..., r:]], -1)


def _exact_append(s, k, v, table, seq, pos):
    """The cache after the append: rows in units of their scale, not rounded to the type (64 bits), and the scales."""
    case, t = s.case, s.case["t"]
    blk, slot = table[seq, pos // t], pos % t
    stored = {name: x.double().clone() for name, x in _cache(s).items()}
    if case["fmt"] == "fp16":
        stored["k"][blk, :, slot], stored["v"][blk, :, slot] = k, v
        return stored
    starts = torch.unique(blk[slot == 0])
    for which, (name, x) in enumerate((("k", k), ("v", v))):
        sc = stored["scales"][:, :, which].clone()
        sc[starts] = 2.0 ** _E_MIN
        most = torch.zeros_like(sc).index_reduce_(0, blk, x.abs().amax(-1), "amax")
        want = torch.exp2(torch.ceil(torch.log2((most / 448).clamp(min=2.0 ** -40))).clamp(_E_MIN, _E_MAX))
        want = torch.where(most > 0, torch.maximum(want, sc), sc)
        changed = torch.unique(blk)
        ratio = torch.ones_like(sc)
        ratio[changed] = (sc / want)[changed]
        ratio[starts] = 1.0
        stored[name] *= ratio[:, :, None, None]
        stored["scales"][changed, :, which] = want[changed]
        stored[name][blk, :, slot] = (x / want[blk][:, :, None]).clamp(-448, 448)
    return stored


def _exact_attention(s, q, k, v, table, lens, new):
    """One sequence and KV head after the other; k, v: the stored values of the whole cache."""
    case, t = s.case, s.case["t"]
    h, g, d = case["h"], case["g"], case["d"]
    out = torch.empty((q.shape[0], h * g, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((q.shape[0], h * g), dtype=torch.float64, device="cuda")
    row = 0
    for i, (n, c) in enumerate(zip(lens, new)):
        n, c = int(n), int(c)
        at = torch.arange(n, device="cuda")
        blk = table[i, at // t].long()
        for head in range(h):
            ki, vi = (x(blk, head, at % t) for x in (k, v))
            for a in range(0, c, 1024):
                b = min(c, a + 1024)
                x = q[row + a:row + b, head * g:(head + 1) * g].double().reshape((b - a) * g, d) @ ki.T.contiguous() / math.sqrt(d)
                sees = torch.arange(n - c + a + 1, n - c + b + 1, device="cuda").repeat_interleave(g)
                x.masked_fill_(at[None] >= sees[:, None], -math.inf)
                lse[row + a:row + b, head * g:(head + 1) * g] = torch.logsumexp(x, 1).view(b - a, g)
                out[row + a:row + b, head * g:(head + 1) * g] = (torch.softmax(x, 1) @ vi).view(b - a, g, d)
        row += c
    return out, lse


def exact(case, seed):
    if case["kind"] == "tables" or work(case)["flops"] > 2e12:
        return None
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_rotation(case, s.x, s.pos, case["inverse"])
    table = s.table.long()
    held, new = _seeded_lens(case, seed)
    got = {}
    if case["kind"] == "step":  # (one new token each: at most one new block, the next of the list where a block begins)
        begins = held % case["t"] == 0
        which = torch.from_numpy(np.flatnonzero(begins)).cuda()
        table[which, torch.from_numpy(held[begins] // case["t"]).cuda()] = s.ids[:int(begins.sum())].long()
    if case["kind"] in ("append", "step"):
        got["q"] = _exact_rotation(case, s.q, s.pos)
        stored = _exact_append(s, _exact_rotation(case, s.k, s.pos), s.v.double(), table, s.seq.long(), s.pos.long())
        got.update(stored)
        if case["kind"] == "append":
            return got
        # attention reads what is stored, in the cache's and the queries' types
        codes = {x: stored[x].float().to(torch.float8_e4m3fn) for x in "kv"}
        q, scales = got["q"].half(), stored["scales"]
    else:
        codes, q = _cache(s), s.q
        scales = codes["scales"].double()

    def rows(x, which):
        return lambda blk, head, slot: x.view(torch.uint8)[blk, head, slot].view(torch.float8_e4m3fn).double() * scales[blk, head, which, None]

    got["out"], got["lse"] = _exact_attention(s, q, rows(codes["k"], 0), rows(codes["v"], 1), table, held + new, new)
    if case["kind"] == "step":
        got.update(dict.fromkeys(("table", "seq_lens", "q_offsets", "seq_idx", "pos", "slots")))
    return got
