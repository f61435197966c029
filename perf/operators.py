"""Cases and plain forms of the paged KV cache held in 4 bits: append + gather, attention, compact, fork.

A cached token holds, for each KV head, d key and d value channels in blocks of 16: an e2m1 code for each channel and an
e4m3 scale for each block; the value is code * scale * 2^exp with one exponent for each KV head.  A page holds `ps` tokens
of all KV heads as [H_kv][ps / 16] groups of 16 tokens, a group as [16][d/2] key codes, [16][d/16] key scales, [16][d/2]
value codes, [16][d/16] value scales (18 d bytes; even channels in the low half of a byte).  A map says which pages a
sequence has: refs [n_pages] (0: free), table [n_seqs][max_pages], lens [n_seqs].
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------ cases
def _attend(name, n, lo, hi, nq_lo, nq_hi, H, Hkv, d, ps, dtype, out, mix):
    return {"name": name, "op": "attend", "n": n, "lo": lo, "hi": hi, "nq_lo": nq_lo, "nq_hi": nq_hi, "H": H, "Hkv": Hkv,
            "d": d, "ps": ps, "dtype": dtype, "out": out, "mix": mix}


def _store(name, n, lo, hi, new_lo, new_hi, Hkv, d, ps, dtype, mix):
    return {"name": name, "op": "store", "n": n, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "Hkv": Hkv, "d": d,
            "ps": ps, "dtype": dtype, "mix": mix}


def _compact(name, n, lo, hi, budget, Hkv, d, ps, mix):
    return {"name": name, "op": "compact", "n": n, "lo": lo, "hi": hi, "budget": budget, "Hkv": Hkv, "d": d, "ps": ps, "mix": mix}


def _fork(name, n, lo, hi, ps, width, ended, mix):
    return {"name": name, "op": "fork", "n": n, "lo": lo, "hi": hi, "ps": ps, "width": width, "ended": ended, "mix": mix}


def listed():
    return [
        # one sequence at a budget of 512, one token: the smallest call, all latency
        _attend("attend_one_token", 1, 513, 513, 1, 1, 32, 8, 128, 64, "bf16", "bf16", 1),
        # the smallest head shape (4 heads on one KV head, d = 64), three sequences of odd lengths, fp16
        _attend("attend_small_heads", 3, 101, 1024, 1, 1, 4, 1, 64, 16, "f16", "f16", 2),
        # a decode step of one layer for a batch of 32 whose sequences are at or below a budget of 2048
        _attend("attend_budget_batch", 32, 1500, 2049, 1, 1, 32, 8, 128, 64, "bf16", "bf16", 3),
        # a decode step over a few very long caches
        _attend("attend_long", 4, 100001, 131072, 1, 1, 32, 8, 128, 128, "bf16", "bf16", 4),
        # drafted tokens checked in one call (1 to 5 of them), 7 query heads on a KV head, float32 outputs
        _attend("attend_drafts", 8, 9000, 16384, 1, 5, 28, 4, 128, 32, "bf16", "f32", 5),
        # a prompt's chunk of 2048 tokens behind 14 K cached ones
        _attend("attend_chunk", 1, 16384, 16384, 2048, 2048, 32, 8, 128, 64, "bf16", "bf16", 6),
        # one new token for each of 32 sequences, read back as the layer would for its evicted entries
        _store("store_decode", 32, 100, 2100, 1, 1, 8, 128, 64, "bf16", 7),
        # four prompts of ragged lengths at once
        _store("store_prompts", 4, 0, 3000, 2001, 8192, 8, 128, 64, "f16", 8),
        # one layer's eviction to the budget of 2048 after an interval of 128 tokens
        _compact("compact_interval", 32, 2176, 2176, 2048, 8, 128, 64, 9),
        # 16 long sequences cut down to a budget of 8192
        _compact("compact_long", 16, 10000, 32768, 8192, 8, 128, 128, 10),
        # a beam step of 4 sequences x 4 beams
        _fork("fork_beams", 16, 200, 1500, 32, 4, 0.1, 11),
        # the rows of 32 layers x 32 sequences reordered and freed in one call
        _fork("fork_all_layers", 1024, 2000, 16384, 64, 4, 0.1, 12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "store", "compact", "fork"])
    ps = rng.choice([16, 32, 64, 128])
    mix = rng.randrange(1 << 30)
    H, Hkv, d = rng.choice([(32, 8, 128), (28, 4, 128), (4, 1, 64), (16, 4, 64), (8, 8, 128), (32, 2, 128), (8, 2, 256), (16, 8, 256)])
    n = _log(rng, 1, 64)
    if op == "attend":
        nq = rng.choice([1, 1, _log(rng, 2, 9), _log(rng, 10, 2048)])
        n = min(n, 64 if nq == 1 else 16 if nq < 10 else 2)
        # no more than the long case has in bytes, nor than the chunk case in products
        hi = _log(rng, 1, min(131072, 500000 * 8 * 128 // (n * Hkv * d), 16384 * 2048 * 32 * 128 // (n * nq * H * d)))
        dtype = rng.choice(["bf16", "f16"])
        return _attend("", n, max(1, hi // rng.choice([1, 2, 20])), hi, max(1, nq // rng.choice([1, 3])), nq, H, Hkv, d, ps, dtype,
                       rng.choice([dtype, dtype, "f32"]), mix)
    if op == "store":
        new = _log(rng, 1, min(8192, 24000 * 8 * 128 // (n * Hkv * d)))
        return _store("", n, 0, _log(rng, 1, 3000), max(1, new // rng.choice([1, 2, 10])), new, Hkv, d, ps, rng.choice(["bf16", "f16"]), mix)
    if op == "compact":
        hi = _log(rng, 8, min(32768, 16 * 32768 * 8 * 128 // (n * Hkv * d)))
        return _compact("", n, max(1, hi // rng.choice([1, 2])), hi, _log(rng, 4, hi), Hkv, d, ps, mix)
    width = rng.choice([1, 2, 4, 8])
    n = width * _log(rng, 1, 1024 // width)
    hi = _log(rng, 10, 16384)
    return _fork("", n, max(1, hi // rng.choice([1, 2, 8])), hi, ps, width, rng.choice([0.0, 0.1, 0.5]), mix)


def _between(case, lo, hi, salt, count=None):
    """Ragged sizes of a case, the same ones for every seed (the largest is `hi` itself)."""
    r = np.random.RandomState((case["mix"] * 7 + salt) % (1 << 31))
    v = r.randint(lo, hi + 1, count or case["n"]).astype(np.int64)
    v[r.randint(len(v))] = hi
    return v


def _lens(case):
    return _between(case, case["lo"], case["hi"], 1)


def _queries(case, lens):
    return np.minimum(_between(case, case["nq_lo"], case["nq_hi"], 2), lens)


def work(case):
    lens = _lens(case)
    row = 1.125 * case.get("d", 0) * case.get("Hkv", 0)  # bytes of one cached token
    if case["op"] == "attend":
        nq = _queries(case, lens)
        q = float(nq.sum()) * case["H"] * case["d"]
        pairs = float((nq * (lens - nq) + nq * (nq + 1) // 2).sum())
        return {"bytes": float(lens.sum()) * row + q * (2 + TYPES[case["out"]].itemsize) + 4 * float(nq.sum()) * case["H"],
                "flops": 4.0 * case["d"] * case["H"] * pairs}
    if case["op"] == "store":  # tokens in, codes out; codes in, values out
        t = float(_between(case, case["new_lo"], case["new_hi"], 3).sum())
        return {"bytes": 2 * t * (row + 4.0 * case["Hkv"] * case["d"])}
    if case["op"] == "compact":
        moved = np.where(lens > case["budget"], case["budget"], 0)
        return {"bytes": 2 * float(moved.sum()) * row + float(lens.sum())}
    pages = float((-(-lens // case["ps"])).sum())
    return {"bytes": 4 * (2 * pages + 2 * _n_pages(case, lens) + 3.0 * case["n"])}


# ------------------------------------------------------------------ inputs
def _n_pages(case, lens):
    """Pages of the pool: what the sequences hold, what the call adds, and a few more."""
    ps = case["ps"]
    held = int((-(-lens // ps)).sum())
    if case["op"] == "store":
        held += int((-(-_between(case, case["new_lo"], case["new_hi"], 3) // ps)).sum()) + 2 * len(lens)
    if case["op"] == "compact":
        held += int((-(-np.minimum(lens, case["budget"]) // ps)).sum())
    return held + 5


def _pages_of(rng, lens, ps, max_pages, n_pages):
    """Shuffled pages dealt to the sequences: table (-1 where there is none) and refs."""
    table = np.full((len(lens), max_pages), -1, np.int32)
    has = np.arange(max_pages)[None, :] < (-(-lens // ps))[:, None]
    ids = rng.permutation(n_pages)[:int(has.sum())]
    table[has] = ids
    refs = np.zeros(n_pages, np.int32)
    refs[ids] = 1
    return table, refs


def _share_tails(table, refs, lens, ps):
    """Every third sequence hands its pages to the next one, as after a fork."""
    for i in range(0, len(lens) - 1, 3):
        refs[table[i + 1][table[i + 1] >= 0]] -= 1
        table[i + 1], lens[i + 1] = table[i], lens[i]
        refs[table[i][table[i] >= 0]] += 1


def _parts(pool, Hkv, d, ps):
    """The pool's bytes as (key codes, key scales, value codes, value scales), each [n_pages][Hkv][ps / 16][16][bytes]."""
    g = pool.view(-1, Hkv, ps // 16, 18 * d)
    cut = lambda a, b, w: g[..., a * d:b * d].unflatten(-1, (16, w))  # noqa: E731
    return cut(0, 8, d // 2), cut(8, 9, d // 16), cut(9, 17, d // 2), cut(17, 18, d // 16)


def _two(exp):
    """2^exp in 64 bits, exactly."""
    return (exp.long() + 1023 << 52).view(torch.float64)


def _cuts(x, edges):
    """How many edges each value has passed; a value on an edge goes to the even side."""
    n = torch.bucketize(x, edges)
    return n + ((n % 2 == 1) & (x == edges[n.clamp(max=len(edges) - 1)]))


def _quantise(x, exp):
    """[..., Hkv, d] -> code bytes [..., Hkv, d/2], scale bytes [..., Hkv, d/16] (in 64 bits: a value next to an edge counts)."""
    x = x.double() * _two(-exp)[:, None]
    b = x.unflatten(-1, (-1, 16))
    s = (b.abs().amax(-1) / 6).clamp(max=448.0).float().to(torch.float8_e4m3fn)
    v = s.double()[..., None]
    y = torch.where(v > 0, b.abs() / v, 0.0)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device=x.device)
    code = (_cuts(y, edges) + 8 * (b < 0)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, s.view(torch.uint8)


def _write_rows(pool, row, k, v, k_exp, v_exp, Hkv, d, ps):
    """Tokens k, v [T][Hkv][d] to the pool's rows (page * ps + slot)."""
    page, group, at = row // ps, row % ps // 16, row % 16
    kc, ks, vc, vs = _parts(pool, Hkv, d, ps)
    kc[page, :, group, at], ks[page, :, group, at] = _quantise(k, k_exp)
    vc[page, :, group, at], vs[page, :, group, at] = _quantise(v, v_exp)


def _tokens(gen, t, Hkv, d, dtype):
    """Keys with a few strong channels, values without."""
    k = torch.randn((t, Hkv, d), generator=gen, device=DEV)
    v = torch.randn((t, Hkv, d), generator=gen, device=DEV) * 0.3
    gain = 1 + 4 * (torch.rand((Hkv, d), generator=gen, device=DEV) < 0.05)
    return (k * gain).to(dtype), v.to(dtype)


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).to(DEV)


def _starts(counts):
    return _ints(np.concatenate([[0], np.cumsum(counts)]))


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 31))
    lens, ps, op = _lens(case), case["ps"], case["op"]
    n_pages = _n_pages(case, lens)
    longest = int(lens.max()) + (case["new_hi"] if op == "store" else 0)
    max_pages = -(-longest // ps)
    table, refs = _pages_of(rng, lens, ps, max_pages, n_pages)
    s = {"op": op, "ps": ps, "n": len(lens), "n_pages": n_pages, "max_pages": max_pages}
    if op == "fork":
        s |= {"Hkv": 1, "d": 64, "pool": torch.zeros(n_pages * ps * 72, dtype=torch.uint8, device=DEV)}
        first = np.arange(len(lens)) // case["width"] * case["width"]
        parent = first + rng.randint(0, case["width"], len(lens))
        parent[rng.rand(len(lens)) < case["ended"]] = -1
        s["parent"] = _ints(parent)
    else:
        Hkv, d = case["Hkv"], case["d"]
        s |= {"Hkv": Hkv, "d": d, "k_exp": _ints(rng.randint(-1, 2, Hkv)), "v_exp": _ints(rng.randint(-4, -1, Hkv))}
        s["pool"] = torch.zeros(n_pages * ps * Hkv * d * 9 // 8, dtype=torch.uint8, device=DEV)
        every = _ints(np.nonzero(refs)[0]).long()[:, None] * ps + torch.arange(ps, device=DEV)
        step = max(1, (1 << 24) // (Hkv * d * ps))
        for at in range(0, len(every), step):  # what the pages hold already
            rows = every[at:at + step].reshape(-1)
            _write_rows(s["pool"], rows, *_tokens(gen, len(rows), Hkv, d, torch.bfloat16), s["k_exp"], s["v_exp"], Hkv, d, ps)
    if op == "attend":
        nq = _queries(case, lens)
        q = torch.randn((int(nq.sum()), case["H"], d), generator=gen, device=DEV) * 1.2
        s |= {"q": q.to(TYPES[case["dtype"]]), "cu": _starts(nq), "max_q": int(nq.max()), "out": TYPES[case["out"]], "longest": longest}
    if op == "store":
        _share_tails(table, refs, lens, ps)
        new = _between(case, case["new_lo"], case["new_hi"], 3)
        s["k"], s["v"] = _tokens(gen, int(new.sum()), Hkv, d, TYPES[case["dtype"]])
        s |= {"cu": _starts(new), "slots": _ints(np.concatenate([np.arange(a, a + b) for a, b in zip(lens, new)]))}
    if op == "compact":
        order = torch.rand((len(lens), longest), generator=gen, device=DEV)
        order[:, :4] = -1.0  # the first tokens stay
        order[torch.arange(longest, device=DEV) >= _ints(lens)[:, None]] = 2.0
        s["keep"] = (order.argsort(1).argsort(1) < case["budget"]).to(torch.uint8)
    s |= {"refs": _ints(refs), "table": _ints(table), "lens": _ints(lens)}
    if op != "attend":
        s |= {"refs_to": torch.zeros_like(s["refs"]), "table_to": torch.full_like(s["table"], -1), "lens_to": torch.zeros_like(s["lens"])}
    return s


# ------------------------------------------------------------------ plain forms
def _read_rows(s, row):
    """float32 keys and values [..., Hkv, d] of the pool's rows."""
    ps, page, group, at = s["ps"], row // s["ps"], row % s["ps"] // 16, row % 16
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=DEV)

    def values(code, scale, exp):
        code, scale = code[page, :, group, at], scale[page, :, group, at]
        x = level[torch.stack([code & 15, code >> 4], -1).flatten(-2).int()].unflatten(-1, (-1, 16))
        return (x * scale.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2) * _two(exp).float()[:, None]

    kc, ks, vc, vs = _parts(s["pool"], s["Hkv"], s["d"], ps)
    return values(kc, ks, s["k_exp"]), values(vc, vs, s["v_exp"])


def _plain_attend(s):
    t, H, d = s["q"].shape
    n, Hkv, longest, nq = s["n"], s["Hkv"], s["longest"], s["max_q"]
    slot = torch.arange(longest, device=DEV)
    row = s["table"][:, slot // s["ps"]].clamp(min=0).long() * s["ps"] + slot % s["ps"]
    k, v = _read_rows(s, row)                                      # [n, longest, Hkv, d]
    count = s["cu"].diff()
    tok = s["cu"][:-1, None] + torch.arange(nq, device=DEV)
    q = s["q"].float()[tok.clamp(max=t - 1).long()].unflatten(2, (Hkv, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    x = q @ k.permute(0, 2, 3, 1) * (1 / math.sqrt(d))             # [n, Hkv, nq * G, longest]
    sees = s["lens"][:, None] - count[:, None] + torch.arange(1, nq + 1, device=DEV)
    hidden = slot >= sees.repeat_interleave(H // Hkv, 1)[:, None, :, None]
    x = x.masked_fill_(hidden, -math.inf)
    most = x.amax(-1, keepdim=True).clamp(min=-3e38)
    p = x.sub_(most).exp_()
    total = p.sum(-1, keepdim=True)
    o = p @ v.permute(0, 2, 1, 3) / total
    lse = (most + total.log())[..., 0]
    at = torch.arange(t, device=DEV)
    seq = torch.searchsorted(s["cu"], at.int(), right=True) - 1
    j = at - s["cu"][seq]
    back = lambda y: y.unflatten(2, (nq, -1))[seq, :, j].flatten(1, 2)  # noqa: E731
    return {"o": back(o).to(s["out"]), "lse": back(lse)}


def _hand_out(s, need, held, kept, total):
    """Pages for sequences that hold `held` of them, keep the first `kept` and need `need` more (`total` in the end): the
    table and refs after it, the lowest free pages first, in order of sequence."""
    page = torch.arange(s["max_pages"], device=DEV)
    free = torch.sort((s["refs"] != 0).int(), stable=True).indices
    first = need.cumsum(0) - need
    nth = first[:, None] + page - kept[:, None]
    mine = (page >= kept[:, None]) & (page < total[:, None])
    table = torch.where(mine, free[nth.clamp(0, s["n_pages"] - 1)].int(), torch.where(page < kept[:, None], s["table"], s["table_to"]))
    change = torch.zeros_like(s["refs"]).scatter_add_(0, table.clamp(min=0).flatten().long(), mine.flatten().int())
    lost = (page >= kept[:, None]) & (page < held[:, None])
    return table, s["refs"] + change.scatter_add_(0, s["table"].clamp(min=0).flatten().long(), -lost.flatten().int())


def _plain_store(s):
    ps, lens, new = s["ps"], s["lens"], s["cu"].diff()
    held, total, last = (lens + ps - 1) // ps, (lens + new + ps - 1) // ps, lens // ps
    shared = (lens % ps > 0) & (new > 0) & (s["refs"][s["table"].gather(1, last.clamp(max=s["max_pages"] - 1)[:, None].long())[:, 0].clamp(min=0)] > 1)
    kept = held - shared.int()
    table, refs = _hand_out(s, total - kept, held, kept, total)
    at = last.clamp(max=s["max_pages"] - 1)[:, None].long()
    fresh = table.gather(1, at).long()  # the page of the first new token (each sequence has one)
    slot = torch.arange(ps, device=DEV)
    copied = shared[:, None] & (slot < (lens % ps)[:, None])
    into, out_of = fresh * ps + slot, torch.where(copied, s["table"].gather(1, at).long(), fresh) * ps + slot
    for part in _parts(s["pool"], s["Hkv"], s["d"], ps):
        part[into // ps, :, slot // 16, slot % 16] = part[out_of // ps, :, slot // 16, slot % 16]
    seq = torch.searchsorted(s["cu"], torch.arange(len(s["k"]), device=DEV, dtype=torch.int32), right=True) - 1
    row = table[seq, s["slots"] // ps].long() * ps + s["slots"] % ps
    _write_rows(s["pool"], row, s["k"], s["v"], s["k_exp"], s["v_exp"], s["Hkv"], s["d"], ps)
    k, v = _read_rows(s, row)
    return {"k": k.to(s["k"].dtype), "v": v.to(s["v"].dtype), "table": table, "refs": refs, "lens": lens + new}


def _plain_compact(s):
    ps, lens = s["ps"], s["lens"]
    slot = torch.arange(s["keep"].shape[1], device=DEV)
    here = slot < lens[:, None]
    keep = here & (s["keep"] != 0)
    count = keep.sum(1).int()
    hole = torch.where(here & ~keep, slot, lens[:, None]).amin(1).int()
    held, total = (lens + ps - 1) // ps, (count + ps - 1) // ps
    kept = torch.where(hole == lens, held, hole // ps)
    table, refs = _hand_out(s, total - kept, held, kept, total)
    source = torch.sort((~keep).int(), stable=True).indices  # survivors first, in order
    moves = (slot >= kept[:, None] * ps) & (slot < count[:, None])
    # a slot without a move copies slot 0 of its sequence's first page onto itself, or page 0 where there is none
    still = s["table"][:, :1].clamp(min=0).long() * ps
    into = torch.where(moves, table[:, slot // ps].long() * ps + slot % ps, still)
    out_of = torch.where(moves, s["table"].gather(1, source // ps).long() * ps + source % ps, still)
    for part in _parts(s["pool"], s["Hkv"], s["d"], ps):
        part[into // ps, :, into % ps // 16, into % 16] = part[out_of // ps, :, out_of % ps // 16, out_of % 16]
    # the pool's bytes are moved as they are: whole numbers, equal or not
    return {"pool": s["pool"], "table": table, "refs": refs, "lens": count}


def _plain_fork(s):
    page, parent = torch.arange(s["max_pages"], device=DEV), s["parent"].long()
    there = parent >= 0
    lens = torch.where(there, s["lens"][parent.clamp(min=0)], 0)
    mine = page < ((lens + s["ps"] - 1) // s["ps"])[:, None]
    table = torch.where(mine, s["table"][parent.clamp(min=0)], s["table_to"])
    before = page < ((s["lens"] + s["ps"] - 1) // s["ps"])[:, None]
    refs = s["refs"].scatter_add(0, table.clamp(min=0).flatten().long(), mine.flatten().int())
    refs = refs.scatter_add(0, s["table"].clamp(min=0).flatten().long(), -before.flatten().int())
    return {"table": table, "refs": refs, "lens": lens}


PLAIN = {"attend": _plain_attend, "store": _plain_store, "compact": _plain_compact, "fork": _plain_fork}


# ------------------------------------------------------------------ the framework's calls
def _handle(s):
    from paper_2605_25475_b200 import binding as im
    s["cache"] = im.KV4Cache(s["n"], s["max_pages"], s["n_pages"], s["Hkv"], s["d"], s["ps"], k_exp=s.get("k_exp"), v_exp=s.get("v_exp"),
                             device=DEV, pool=s["pool"], map=im.KV4Map(s["refs"], s["table"], s["lens"]))
    if "refs_to" in s:
        s["to"] = im.KV4Map(s["refs_to"], s["table_to"], s["lens_to"])


def _calls(s):
    if "cache" not in s:  # the handle that a program keeps
        _handle(s)
    c = s["cache"]
    if s["op"] == "attend":
        o, lse = c.attend(s["q"], s["cu"], s["max_q"], out_f32=s["out"] == torch.float32, return_lse=True)
        return {"o": o, "lse": lse}
    to = {"table": s["table_to"], "refs": s["refs_to"], "lens": s["lens_to"]}
    if s["op"] == "store":
        c.append(s["k"], s["v"], s["cu"], to=s["to"])
        k, v = c.gather(s["slots"], s["cu"], dtype=s["k"].dtype, map=s["to"])
        return {"k": k, "v": v, **to}
    if s["op"] == "compact":
        c.compact(s["keep"], to=s["to"])
        return {"pool": s["pool"], **to}
    c.fork(s["parent"], to=s["to"])
    return to


def run(state):
    return _calls(state) if own else PLAIN[state["op"]](state)


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _powers(e, bias):
    """2^(e - bias) of small whole numbers e."""
    return torch.tensor([2.0 ** (i - bias) for i in range(256)], dtype=torch.float64, device=DEV)[e.long()]


def _e2m1(c):
    e, m = c >> 1 & 3, (c & 1).double()
    return torch.where(e > 0, _powers(e, 1) * (1 + m / 2), m / 2) * torch.where(c > 7, -1.0, 1.0).double()


def _e4m3(c):
    e, m = c >> 3 & 15, (c & 7).double()
    return torch.where(e > 0, _powers(e, 7) * (1 + m / 8), m * 2.0 ** -9)


def _nearest(x, values):
    """The index of the nearest of ascending values; of two as near, the even one."""
    hi = torch.searchsorted(values, x).clamp(1, len(values) - 1)
    up, down = values[hi] - x, x - values[hi - 1]
    return torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)


def _stored(x, exp):
    """What the cache holds for tokens x [T][Hkv][d]."""
    one = _powers(exp + 64, 64)[:, None, None]
    b = x.double().unflatten(-1, (-1, 16)) / one
    scales = _e4m3(torch.arange(127, device=DEV))
    codes = _e2m1(torch.arange(8, device=DEV))
    s = scales[_nearest(b.abs().amax(-1, keepdim=True) / 6, scales)]
    held = codes[_nearest(torch.where(s > 0, b.abs() / s, 0.0), codes)] * s
    return (torch.where(b < 0, -held, held) * one).flatten(-2)


def exact(case, seed):
    if case["op"] not in ("attend", "store"):
        return None  # moves and counts: nothing is computed
    s = prepare(case, seed)
    if case["op"] == "store":
        return {"k": _stored(s["k"], s["k_exp"]), "v": _stored(s["v"], s["v_exp"]), "table": None, "refs": None, "lens": None}
    Hkv, d, ps, H = s["Hkv"], s["d"], s["ps"], case["H"]
    page = s["pool"].view(-1, Hkv, ps // 16, 2, 9 * d)
    lens, cu, table = s["lens"].tolist(), s["cu"].tolist(), s["table"].long()
    o, lse = [], []
    for i, n in enumerate(lens):
        a, b = cu[i], cu[i + 1]
        rows = page[table[i, :-(-n // ps)]].transpose(0, 1).flatten(1, 2)                 # [Hkv, groups, 2, 9 d]
        sees = torch.arange(n - (b - a) + 1, n + 1, device=DEV)
        out, total = [], []
        for h in range(Hkv):
            held = []
            for which, exp in ((0, s["k_exp"]), (1, s["v_exp"])):
                byte = rows[h, :, which].int()
                code = byte[:, :8 * d].reshape(-1, d // 2)[:n]
                scale = _e4m3(byte[:, 8 * d:].reshape(-1, d // 16)[:n])
                x = torch.stack([_e2m1(code % 16), _e2m1(code // 16)], 2).reshape(n, d // 16, 16)
                held.append((x * scale[..., None]).reshape(n, d) * 2.0 ** float(exp[h]))
            q = s["q"][a:b, h * (H // Hkv):(h + 1) * (H // Hkv)].double()                   # [nq, G, d]
            got, sums = [], []
            for at in range(0, b - a, 256):
                x = q[at:at + 256] @ held[0].T / math.sqrt(d)
                x = torch.where(torch.arange(n, device=DEV) < sees[at:at + 256, None, None], x, -math.inf)
                sums.append(torch.logsumexp(x, -1))
                got.append(torch.exp(x - sums[-1][..., None]) @ held[1])
            out.append(torch.cat(got))
            total.append(torch.cat(sums))
        o.append(torch.cat(out, 1))
        lse.append(torch.cat(total, 1))
    return {"o": torch.cat(o), "lse": torch.cat(lse)}
