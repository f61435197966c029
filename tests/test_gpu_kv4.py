"""The paged 4-bit KV cache (im_kv4_*) against tests/kv4_reference.py: the maps and what the cache holds exactly, attention
within a bound derived below."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def im():
    from paper_2605_25475_b200 import binding
    return binding


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda:0")


def starts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)


class Pair:
    """The library's cache and the reference, driven together."""

    def __init__(self, im, n_seqs, max_pages, n_pages, Hkv, d, ps, seed=0, exps=True):
        self.rng = np.random.RandomState(seed)
        ke = self.rng.randint(-2, 3, Hkv) if exps else None
        ve = self.rng.randint(-5, 1, Hkv) if exps else None
        self.im, self.Hkv, self.d = im, Hkv, d
        self.g = im.KV4Cache(n_seqs, max_pages, n_pages, Hkv, d, ps, k_exp=None if ke is None else ints(ke), v_exp=None if ve is None else ints(ve))
        self.g.pool.fill_(0xFF)  # codes -6, scales NaN: what was never written must not be seen
        self.r = ref.Cache(n_seqs, max_pages, n_pages, Hkv, d, ps, ke, ve)

    def tokens(self, n, dtype=BF, spread=1.0):
        k = self.rng.randn(n, self.Hkv, self.d) * spread * np.exp(0.5 * self.rng.randn(n, self.Hkv, 1))
        v = self.rng.randn(n, self.Hkv, self.d) * 0.3
        return (torch.tensor(x, dtype=torch.float32).to(dtype).cuda() for x in (k, v))

    def append(self, counts, dtype=BF, to=None):
        k, v = self.tokens(int(np.sum(counts)), dtype)
        cu = starts(counts)
        self.g.append(k, v, ints(cu), to=to)
        ok = self.r.append(k.double().cpu().numpy(), v.double().cpu().numpy(), cu)
        return ok

    def check(self, map=None):
        m = map or self.g.map
        np.testing.assert_array_equal(m.lens.cpu().numpy(), self.r.lens)
        np.testing.assert_array_equal(m.refs.cpu().numpy(), self.r.refs)
        table = m.table.cpu().numpy()
        for i in range(self.r.n):
            n = self.r.pages(self.r.lens[i])
            np.testing.assert_array_equal(table[i, :n], self.r.table[i, :n], err_msg=f"row {i}")
        k, v = self.g.gather(n_rows=int(self.r.lens.sum()), cu_rows=ints(starts(self.r.lens)), dtype=F32, map=map)
        want = [self.r.kv(i) for i in range(self.r.n)]
        np.testing.assert_array_equal(k.double().cpu().numpy(), np.concatenate([w[0] for w in want]))
        np.testing.assert_array_equal(v.double().cpu().numpy(), np.concatenate([w[1] for w in want]))

    def attend(self, counts, H, dtype=BF, out_f32=False, causal=True, scale=0.0, spread=1.0, stride=None, max_q=None, q=None):
        cu, d = starts(counts), self.d
        T = int(cu[-1])
        if q is None:
            q = torch.tensor(self.rng.randn(T, H, d) * spread, dtype=F32).to(dtype).cuda()
        if stride:
            wide = torch.full((T, stride), float("nan"), dtype=dtype, device="cuda:0")
            wide[:, 8:8 + H * d] = q.view(T, H * d)
            q = wide[:, 8:8 + H * d].unflatten(1, (H, d))
        o, lse = self.g.attend(q, ints(cu), int(max(counts)) if max_q is None else max_q, softmax_scale=scale, causal=causal,
                               out_f32=out_f32, return_lse=True)
        sc = scale or 1 / np.sqrt(d)
        check_attention(self.r, q, cu, sc, causal, o, lse)
        return o, lse


def check_attention(r, q, cu, sc, causal, o, lse):
    """|error| of an output <= half a step of its type + A sum_t p_t |v_t|, where A collects the relative errors of p and of
    the sums.  Scores: products are exact, a sum of d of them in float32 errs by at most (d + 4) 2^-23 of the sum of their
    absolute values (`spread`; any order, truncating adders); the base-2 exponent's argument, formed with a multiply-add from a
    rounded scale, by 4 x 2^-24 of its size, which `spread` bounds too, and exp2 by 2^-22.  p has one error e and the sum that
    divides it has the same: 2 e.  p is kept in f16 for bf16 outputs (2^-11) and in two f16 terms otherwise (2^-20); a p
    below f16's normal range is off by half of f16's smallest step, 2^-25, while the row's largest p is kept as 2^7 and
    the sum that divides is no less: 2^-32 sum_t |v_t|.  Sums over L entries in float32, scaled at most once a tile: (L / 16 + 64)
    2^-22 of the sum of absolute values covers any split."""
    d = q.shape[2]
    qn = q.double().cpu().numpy()
    out, ls, weight, spread, every = r.attend(qn, cu, sc, causal)
    L = max(1, int(r.lens.max()))
    e = ((d + 4) * 2.0 ** -23 + 2.0 ** -22) * spread[..., None] + 2.0 ** -22
    sums = (L / 16 + 64) * 2.0 ** -22
    A = 2 * e + (2.0 ** -11 if o.dtype == BF else 2.0 ** -20) + sums
    half = torch.finfo(o.dtype).eps / 2
    tiny = torch.finfo(o.dtype).tiny * torch.finfo(o.dtype).eps  # below the normal range steps are of this size
    got = o.double().cpu().numpy()
    bound = half * np.abs(out) + (1 + half) * (A * weight + 2.0 ** -32 * every) + tiny
    bad = ~(np.abs(got - out) <= bound)
    assert not bad.any(), f"{bad.sum()} outputs off, worst {np.nanmax(np.abs(got - out) / bound)} of the bound"
    gl = lse.double().cpu().numpy()
    empty = np.isinf(ls)
    np.testing.assert_array_equal(gl[empty], ls[empty])
    assert (got[empty] == 0).all()
    lb = e[..., 0] + sums + 2.0 ** -22 * (1 + np.abs(np.where(empty, 0, ls)))
    assert (np.abs(gl[~empty] - ls[~empty]) <= lb[~empty]).all(), (np.abs(gl[~empty] - ls[~empty]) / lb[~empty]).max()


# ------------------------------------------------------------------ what the cache holds
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_quantiser_is_exact(im, d, dtype):
    """Every block kind: ties of codes and of scales, zeros, single values, tiny and huge ones, all sixteen codes."""
    rng = np.random.RandomState(d)
    n, H = 96, 3
    x = rng.randn(n, H, d)
    x[8:24] = np.round(x[8:24] * 4) / 4 * 2.0 ** rng.randint(-4, 5, (16, H, 1))       # many values on code edges
    x[24:40] = rng.choice([0.0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -5.0, -2.5, -6.0], (16, H, d)) * 2.0 ** rng.randint(-3, 4, (16, H, 1))
    x[40:44] = 0.0
    x[44:52] = 0.0
    x[44:52, :, ::16] = rng.randn(8, H, d // 16)                                        # one value in a block
    x[52:60] *= 2.0 ** -9                                                               # scales in the subnormal range
    x[60:64] *= 2.0 ** -13                                                              # ... that round to 0
    x[64:72] *= 2.0 ** 9                                                                # ... that saturate
    amax = 6 * ref.E4M3[rng.randint(8, 120, (8, H, d // 16))] * rng.choice([1, 1 + 1 / 16, 1 + 1 / 32], (8, H, d // 16))
    x[72:80, :, 5::16] = amax                                                           # on and next to scale edges
    pair = Pair(im, 1, 7, 7, H, d, 16, seed=d)
    k, v = (torch.tensor(a, dtype=F32).to(dtype).cuda() for a in (x, x[::-1].copy()))
    pair.g.append(k, v, ints([0, n]))
    assert pair.r.append(k.double().cpu().numpy(), v.double().cpu().numpy(), [0, n])
    pair.check()
    assert pair.g.status() == 0
    for out in (BF, HF):                                                                # exact in the narrow types too
        a, b = pair.g.gather(n_rows=n, cu_rows=ints([0, n]), dtype=out)
        want = pair.r.kv(0)
        fits = np.abs(want[0]) >= 2.0 ** -24
        np.testing.assert_array_equal(a.double().cpu().numpy()[fits], want[0][fits])
        np.testing.assert_array_equal(b.double().cpu().numpy(), torch.tensor(want[1]).to(out).double().numpy())


def test_values_that_are_not_finite(im):
    pair = Pair(im, 2, 2, 4, 2, 64, 16, exps=False)
    k, v = pair.tokens(5)
    k[1, 0, 3], k[1, 1, 17], v[2, 0, 40], v[4, 1, 0] = float("nan"), float("inf"), -float("inf"), float("nan")
    pair.g.append(k, v, ints([0, 2, 5]))
    assert pair.r.append(k.double().cpu().numpy(), v.double().cpu().numpy(), [0, 2, 5])
    pair.check()
    assert pair.g.status(clear=True) == im.IM_KV4_NONFINITE
    pair.append([3, 0])
    assert pair.g.status() == 0


def test_strided_tokens_and_types(im):
    pair = Pair(im, 3, 4, 12, 2, 128, 32, seed=3)
    qkv = torch.randn(40, 1000 // 8 * 8, device="cuda:0").to(HF)                         # a fused projection's rows
    k, v = qkv[:, 8:264].unflatten(1, (2, 128)), qkv[:, 640:896].unflatten(1, (2, 128))
    cu = [0, 0, 33, 40]
    pair.g.append(k, v, ints(cu))
    assert pair.r.append(k.double().cpu().numpy(), v.double().cpu().numpy(), cu)
    pair.check()


# ------------------------------------------------------------------ maps
@pytest.mark.parametrize("d,ps,Hkv", [(64, 16, 1), (128, 64, 2), (128, 32, 8), (256, 128, 3)])
@pytest.mark.parametrize("apart", [False, True])
def test_append_and_fork_share_until_written(im, d, ps, Hkv, apart):
    n = 5
    pair = Pair(im, n, 6, 40, Hkv, d, ps, seed=ps)
    step = pair.g.map
    rng = pair.rng
    for it in range(6):
        counts = rng.choice([0, 1, 1, 2, ps // 2, ps - 1], n)
        if it == 3:
            counts[:] = 1
        to = im.KV4Map(torch.full_like(step.refs, 77), torch.full_like(step.table, -5), torch.full_like(step.lens, -9)) if apart else None
        before = step.clone()
        k, v = pair.tokens(int(counts.sum()), HF)
        cu = starts(counts)
        pair.g.append(k, v, ints(cu), map=step, to=to)
        assert pair.r.append(k.double().cpu().numpy(), v.double().cpu().numpy(), cu)
        if apart:                                                                       # `from` is as it was, rows behind the pages too
            assert torch.equal(step.refs, before.refs) and torch.equal(step.table, before.table) and torch.equal(step.lens, before.lens)
            for i in range(n):
                assert (to.table[i, pair.r.pages(pair.r.lens[i]):] == -5).all()
            step = to
        pair.check(step)
        parent = rng.randint(-1 if it > 2 else 0, n, n)
        to = im.KV4Map(torch.empty_like(step.refs), torch.full_like(step.table, -5), torch.empty_like(step.lens)) if apart else None
        pair.g.fork(ints(parent), map=step, to=to)
        pair.r.fork(parent)
        step = to if apart else step
        pair.check(step)
    assert pair.g.status() == 0


def test_a_call_that_cannot_be_made_changes_nothing(im):
    pair = Pair(im, 3, 3, 6, 2, 64, 16, seed=9)
    assert pair.append([20, 40, 3])                                                      # all six pages
    pool, m = pair.g.pool.clone(), pair.g.map.clone()

    def same():
        assert torch.equal(pair.g.pool, pool) and all(torch.equal(getattr(m, a), getattr(pair.g.map, a)) for a in ("refs", "table", "lens"))

    assert not pair.append([1, 1, 14])                                                   # one page short
    same()
    assert pair.g.status(clear=True) == im.IM_KV4_NO_PAGES
    assert not pair.append([29, 0, 0])                                                   # a row longer than max_pages
    same()
    assert pair.g.status(clear=True) == im.IM_KV4_NO_PAGES
    k, v = pair.tokens(4)
    for cu in ([0, 2, 1, 4], [-1, 1, 2, 3], [0, 1, 2, 5]):
        pair.g.append(k, v, ints(cu))
        same()
        assert pair.g.status(clear=True) == im.IM_KV4_BAD_MAP
    to = im.KV4Map(torch.empty_like(m.refs), torch.empty_like(m.table), torch.empty_like(m.lens))
    pair.g.append(k, v, ints([0, 0, 0, 4]), to=to)                                       # made: fits the last page
    assert pair.g.status() == 0
    pool = pair.g.pool.clone()                                                           # (the new tokens lie behind the old length)
    pair.g.append(*pair.tokens(40), ints([0, 0, 0, 40]), to=to)                          # not made: `to` is a copy
    assert torch.equal(to.refs, m.refs) and torch.equal(to.lens, m.lens) and pair.g.status(clear=True) == im.IM_KV4_NO_PAGES
    keep = torch.ones(3, 40, dtype=torch.uint8, device="cuda:0")
    keep[:, 0] = 0
    pair.g.compact(keep)                                                                 # survivors need free pages: there are none
    same()
    assert pair.g.status(clear=True) == im.IM_KV4_NO_PAGES
    pair.g.compact(keep[:, :39].contiguous())                                            # a mask shorter than a sequence
    same()
    assert pair.g.status(clear=True) == im.IM_KV4_BAD_MAP
    pair.check()


def test_tokens_outside_cu_belong_to_nobody(im):
    pair = Pair(im, 2, 2, 4, 1, 64, 16)
    k, v = pair.tokens(9)
    k[0, 0, 0], k[8, 0, 0] = float("nan"), float("nan")
    pair.g.append(k, v, ints([1, 4, 8]))
    assert pair.r.append(k.double().cpu().numpy()[1:], v.double().cpu().numpy()[1:], [0, 3, 7])
    pair.check()
    assert pair.g.status() == 0
    q = torch.randn(9, 2, 64, device="cuda:0").to(BF)
    out = torch.full((9, 2, 64), 7.0, dtype=BF, device="cuda:0")
    pair.g.attend(q, ints([2, 3, 5]), 2, out=out)
    assert (out[:2] == 7).all() and (out[5:] == 7).all() and not (out[2:5] == 7).any()


def test_fork_with_bad_parents(im):
    pair = Pair(im, 4, 3, 12, 1, 64, 16)
    pair.append([5, 17, 33, 2])
    pair.g.fork(ints([4, 1, -2, 0]))
    pair.r.fork([0, 1, 2, 0])
    pair.check()
    assert pair.g.status() == im.IM_KV4_BAD_MAP


@pytest.mark.parametrize("d,ps,Hkv", [(64, 16, 2), (128, 64, 2), (256, 32, 1), (128, 128, 9)])
@pytest.mark.parametrize("apart", [False, True])
def test_compact(im, d, ps, Hkv, apart):
    n = 7
    pair = Pair(im, n, 5, 80, Hkv, d, ps, seed=d + ps)
    rng = pair.rng
    assert pair.append([0, 1, ps, ps + 1, 3 * ps - 5, 5 * ps, 2 * ps + 7])
    pair.g.fork(ints([0, 1, 2, 3, 4, 5, 5]))                                             # the last row shares the sixth's pages
    pair.r.fork([0, 1, 2, 3, 4, 5, 5])
    pair.g.fork(ints([0, 1, 2, 3, 4, 4, 5]))
    pair.r.fork([0, 1, 2, 3, 4, 4, 5])
    stride = 5 * ps + (3 if apart else 0)                                                # rows that are not 16-byte aligned too
    keep = (rng.rand(n, stride) < 0.6).astype(np.uint8) * rng.randint(1, 256, (n, stride)).astype(np.uint8)
    keep[3] = 0                                                                          # nothing survives
    keep[4] = 200                                                                        # nothing is dropped
    keep[6, :2 * ps + 3] = 1                                                             # two whole pages stay shared
    to = im.KV4Map(torch.empty_like(pair.g.map.refs), pair.g.map.table.clone(), torch.empty_like(pair.g.map.lens)) if apart else None
    pair.g.compact(torch.tensor(keep, device="cuda:0"), to=to)
    assert pair.r.compact(keep)
    pair.check(to)
    assert pair.g.status() == 0


def test_compact_takes_the_selections_mask(im):
    """im_topb_select's keep goes straight in; the dropped entries are read back first, as a memory write needs them."""
    pair = Pair(im, 3, 4, 24, 2, 128, 64, seed=5)
    assert pair.append([200, 200, 200])
    scores = torch.randn(3, 200, device="cuda:0")
    pos = torch.arange(200, dtype=torch.int32, device="cuda:0").repeat(3, 1)
    keep, gone = im.im_topb_select(scores, pos, 129, 4)
    out = torch.nonzero(keep == 0)[:, 1].to(torch.int32)
    k, v = pair.g.gather(out, ints([0, 71, 142, 213]), dtype=F32)
    for i in range(3):
        K, V = pair.r.kv(i)
        rows = out[71 * i:71 * (i + 1)].cpu().numpy()
        np.testing.assert_array_equal(k[71 * i:71 * (i + 1)].double().cpu().numpy(), K[rows])
        np.testing.assert_array_equal(v[71 * i:71 * (i + 1)].double().cpu().numpy(), V[rows])
    pair.g.compact(keep)
    assert pair.r.compact(keep.cpu().numpy())
    pair.check()


def test_gather_of_entries_that_are_not_there(im):
    pair = Pair(im, 2, 2, 4, 2, 64, 16)
    pair.append([3, 20])
    slots = ints([0, 3, -1, 19, 20, 1 << 30, 2])
    k, v = pair.g.gather(slots, ints([0, 3, 7]), dtype=BF)
    K0, K1 = pair.r.kv(0)[0], pair.r.kv(1)[0]
    zero = np.zeros_like(K0[0])
    np.testing.assert_array_equal(k.double().cpu().numpy(), np.stack([K0[0], zero, zero, K1[19], zero, zero, K1[2]]))
    assert (v[[1, 2, 4, 5]] == 0).all()


# ------------------------------------------------------------------ attention
SHAPES = [(32, 8, 128), (4, 1, 64), (28, 4, 128), (8, 8, 64), (32, 2, 128), (6, 2, 256), (40, 2, 128), (9, 1, 64), (24, 2, 256)]


@pytest.mark.parametrize("H,Hkv,d", SHAPES)
@pytest.mark.parametrize("ps", [16, 64])
@pytest.mark.parametrize("dtype,f32", [(BF, False), (HF, False), (BF, True)])
def test_attention_of_one_token(im, H, Hkv, d, ps, dtype, f32):
    lens = [1, 15, 16, 17, 31, 32, 33, 64, 200, 0, 257]
    pair = Pair(im, len(lens), -(-max(lens) // ps), 120, Hkv, d, ps, seed=H + ps)
    assert pair.append(lens)
    o, _ = pair.attend([1] * len(lens), H, dtype, f32)
    again = pair.g.attend(torch.zeros(len(lens), H, d, dtype=dtype, device="cuda:0"), out_f32=f32)  # without cu
    assert again.shape == o.shape and torch.isfinite(again.float()).all() and pair.g.status() == 0


@pytest.mark.parametrize("H,Hkv,d", SHAPES[:6])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("counts", [[2, 1, 0, 5, 3], [9, 4, 1, 17, 33], [40, 0, 75, 1, 12]])
def test_attention_of_several_tokens(im, H, Hkv, d, causal, counts):
    lens = [40, 3, 50, 161, 90]                                                          # the second has fewer entries than queries
    pair = Pair(im, 5, 6, 30, Hkv, d, 32, seed=H + sum(counts))
    assert pair.append(lens)
    pair.attend(counts, H, BF, False, causal)
    pair.attend(counts, H, HF, True, causal, scale=0.05, stride=H * d + 24)
    assert pair.g.status() == 0


@pytest.mark.parametrize("H,Hkv,d,n", [(8, 2, 128, 20011), (4, 1, 64, 33333), (4, 2, 256, 9001)])
def test_attention_over_a_long_cache(im, H, Hkv, d, n):
    pair = Pair(im, 2, -(-n // 128), 320, Hkv, d, 128, seed=1)
    assert pair.append([n, 700])
    pair.attend([1, 1], H, BF)
    pair.attend([3, 1], H, BF, True)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_a_chunk(im, d):
    """A prompt's chunk behind cached tokens, next to a single-token sequence and an empty one."""
    pair = Pair(im, 4, 16, 40, 2, d, 64, seed=2)
    assert pair.append([700, 129, 0, 1000])
    pair.attend([300, 1, 0, 130], 8, BF)
    pair.attend([700, 129, 0, 257], 8, HF, True)
    pair.attend([130, 129, 0, 64], 14, BF, True, causal=False)


@pytest.mark.parametrize("d,dtype", [(128, BF), (128, HF), (64, BF)])
def test_many_rows_agree_with_few_rows_over_a_long_cache(im, d, dtype):
    """The kernel for many query rows against the one for few (max_q chooses it) on 520 tokens x 9000 entries, the reference
    maximum rising all along (keys grow with their position), in fresh memory that holds NaN where nothing was written."""
    n, nq, H, Hkv = 9000, 520, 8, 2
    g = im.KV4Cache(1, -(-n // 64), -(-n // 64), Hkv, d, 64)
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    k, v = (torch.randn(n, Hkv, d, generator=gen, device="cuda:0") for _ in range(2))
    k *= torch.linspace(0.2, 3.0, n, device="cuda:0")[:, None, None]
    cu = ints([0, n])
    g.append(k.to(BF), v.to(BF), cu)
    q = torch.randn(nq, H, d, generator=gen, device="cuda:0").to(dtype)
    cu = ints([0, nq])
    want, wl = g.attend(q, cu, 1, out_f32=True, return_lse=True)
    bound = torch.finfo(dtype).eps / 2 + 2.0 ** -11                                      # of the outputs and of p (for bf16), as above
    for _ in range(4):
        junk = torch.full((1 << 26,), float("nan"), device="cuda:0")
        del junk
        out, lse = g.attend(q, cu, nq, return_lse=True)
        # p >= 0 sums to one over 9000 values of size one: sum p |v| is at most a few units
        assert (out.float() - want).abs().max() <= bound * want.abs().max() + 2.0 ** -11 * v.abs().max()
        assert (lse - wl).abs().max() <= 1e-4 * wl.abs().max()
    assert g.status() == 0


@pytest.mark.parametrize("d,H,n,nq,L", [(64, 2, 1, 40, 70), (128, 4, 2, 24, 130), (256, 2, 1, 33, 100), (256, 8, 3, 200, 300)])
@pytest.mark.parametrize("hint", [1, 2])
def test_a_max_q_too_small_stays_inside_the_workspace(im, monkeypatch, d, H, n, nq, L, hint):
    """The call holds more tiles than its max_q says and its workspace has partial results for: fewer workers share them.  The
    bytes behind the workspace keep their pattern, and the results are right."""
    pair = Pair(im, n, 6, 20, 2, d, 64, seed=6)
    assert pair.append([L] * n)
    ask, seen = pair.g._workspace, []

    def guarded(*a):
        _, nbytes = ask(*a)
        seen.append((torch.full((nbytes + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda:0"), nbytes))
        return seen[-1]

    monkeypatch.setattr(pair.g, "_workspace", guarded)
    for out_f32 in (False, True):
        pair.attend([nq] * n, H, BF, out_f32, max_q=hint)
    assert len(seen) == 2 and all(bool((ws[nbytes:] == 0xA5).all()) for ws, nbytes in seen)
    assert pair.g.status() == 0


@pytest.mark.parametrize("spread", [1e-30, 30.0, 1e4])
def test_attention_of_extreme_queries(im, spread):
    """Queries far outside f16's range, and scores that pick one entry alone."""
    pair = Pair(im, 3, 5, 15, 2, 128, 64, seed=4, exps=False)
    assert pair.append([300, 20, 129])
    pair.attend([1, 2, 1], 8, BF, True, spread=spread)
    pair.attend([1, 2, 90], 8, BF, False, spread=spread)
    q = torch.zeros(3, 8, 128, dtype=BF, device="cuda:0")
    o, lse = pair.attend([1, 1, 1], 8, BF, True, q=q)                                    # all scores equal: the mean of the values
    np.testing.assert_allclose(lse.cpu().numpy(), np.log([[300.0] * 8, [20.0] * 8, [129.0] * 8]), rtol=1e-6)


def test_queries_that_are_not_finite_stay_in_their_rows(im):
    pair = Pair(im, 2, 3, 6, 2, 128, 64, seed=4)
    assert pair.append([100, 100])
    q = torch.randn(4, 8, 128, device="cuda:0").to(BF)
    clean = pair.g.attend(q, ints([0, 2, 4]), 2)
    q[1, 3, 5], q[2, 7, 0] = float("nan"), float("inf")
    got = pair.g.attend(q, ints([0, 2, 4]), 2)
    hurt = torch.zeros(4, 8, dtype=torch.bool, device="cuda:0")
    hurt[1, 3] = hurt[2, 7] = True
    assert torch.equal(got[~hurt], clean[~hurt]) and torch.isnan(got[hurt]).all()


@pytest.mark.parametrize("nq", [1, 9])
def test_bad_pages_are_skipped_and_flagged(im, nq):
    pair = Pair(im, 2, 4, 8, 1, 64, 16, exps=False)
    assert pair.append([50, 20])
    q = torch.randn(2 * nq, 4, 64, device="cuda:0").to(BF)
    cu = ints([0, nq, 2 * nq])
    m = pair.g.map.clone()
    m.table[0, 1] = 8                                                                    # past the pool
    m.table[1, 0] = -3
    o, lse = pair.g.attend(q, cu, nq, return_lse=True, out_f32=True, causal=False, map=m)
    assert pair.g.status(clear=True) == im.IM_KV4_BAD_MAP
    r = pair.r
    for i, rows in ((0, list(range(16)) + list(range(32, 50))), (1, list(range(16, 20)))):
        K, V = r.kv(i)
        s = np.einsum("qhd,td->qht", q[nq * i:nq * i + nq].double().cpu().numpy(), K[rows, 0]) / 8
        p = np.exp(s - s.max(2, keepdims=True))
        np.testing.assert_allclose(o[nq * i:nq * i + nq].double().cpu().numpy(), p @ V[rows, 0] / p.sum(2, keepdims=True), rtol=1e-4, atol=1e-5)
    m.lens[0], m.lens[1] = -5, 1000                                                      # lengths out of range: none, and the row's capacity
    o = pair.g.attend(q, cu, nq, map=m)
    assert (o[:nq] == 0).all()


# ------------------------------------------------------------------ together
def test_a_run_of_all_calls_captured_and_replayed(im):
    """Decode steps as a serving loop makes them: append, attend, evict every few tokens, fork; the step is one graph."""
    n, H, Hkv, d, ps = 4, 8, 2, 128, 16
    pair = Pair(im, n, 12, 80, Hkv, d, ps, seed=8)
    assert pair.append([50, 51, 60, 3])
    g = pair.g
    k = torch.zeros(n, Hkv, d, dtype=BF, device="cuda:0")
    v, q = torch.zeros_like(k), torch.zeros(n, H, d, dtype=BF, device="cuda:0")
    parent = ints(np.arange(n))
    keep = torch.ones(n, 12 * ps, dtype=torch.uint8, device="cuda:0")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        g.append(k, v)
        out, lse = g.attend(q, out_f32=True, return_lse=True)
        g.compact(keep)
        g.fork(parent)
    pair.check()                                                                         # capture alone changes nothing
    for step in range(20):
        kn, vn = pair.tokens(n)
        qn = torch.randn(n, H, d, device="cuda:0").to(BF)
        par = np.arange(n) if step % 3 else pair.rng.randint(0, n, n)
        kp = np.ones((n, 12 * ps), np.uint8) if step % 4 else (pair.rng.rand(n, 12 * ps) < 0.8).astype(np.uint8)
        k.copy_(kn), v.copy_(vn), q.copy_(qn), parent.copy_(ints(par)), keep.copy_(torch.tensor(kp))
        graph.replay()
        assert pair.r.append(kn.double().cpu().numpy(), vn.double().cpu().numpy(), np.arange(n + 1))
        check_attention(pair.r, qn, np.arange(n + 1), 1 / np.sqrt(d), True, out, lse)
        assert pair.r.compact(kp)
        pair.r.fork(par)
        pair.check()
    assert g.status() == 0


def test_two_streams_and_rows_of_one_cache(im):
    """The rows of two layers of one pool: attention of both at once on two streams, each with its own workspace."""
    pair = Pair(im, 8, 11, 90, 2, 128, 64, seed=6)
    assert pair.append([500, 400, 300, 200, 640, 33, 1, 64])
    q = torch.randn(8, 8, 128, device="cuda:0").to(BF)
    want = pair.g.attend(q)
    views = [pair.g.rows(0, 4), pair.g.rows(4, 8)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for it in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got.append((i, views[i].attend(q[4 * i:4 * i + 4])))
    torch.cuda.synchronize()
    for i, o in got:
        assert torch.equal(o, want[4 * i:4 * i + 4])
    k, v = pair.tokens(4)                                                                # an append to one layer's rows
    views[1].append(k, v)
    torch.cuda.synchronize()
    assert pair.r.append(k.double().cpu().numpy(), v.double().cpu().numpy(), [0, 0, 0, 0, 0, 1, 2, 3, 4])
    pair.check()


def test_results_do_not_depend_on_the_run(im):
    pair = Pair(im, 3, 40, 120, 2, 128, 64, seed=7)
    assert pair.append([2500, 1111, 7])
    q = torch.randn(3, 8, 128, device="cuda:0").to(BF)
    first = pair.g.attend(q, out_f32=True)
    for _ in range(10):
        assert torch.equal(first, pair.g.attend(q, out_f32=True))


def test_offsets_past_32_bits(im):
    """A pool of more than 4 GiB: the pages in use are the last ones."""
    Hkv, d, ps = 8, 128, 128
    n_pages = (1 << 32) // im.im_kv4_page_bytes(Hkv, d, ps) + 40
    g = im.KV4Cache(1, 8, n_pages, Hkv, d, ps)
    g.map.refs[:n_pages - 8] = 1                                                         # somebody holds all the others
    rng = np.random.RandomState(0)
    k, v = (torch.tensor(rng.randn(600, Hkv, d), dtype=F32).to(BF).cuda() for _ in range(2))
    g.append(k, v, ints([0, 600]))
    r = ref.Cache(1, 8, 8, Hkv, d, ps)
    assert r.append(k.double().cpu().numpy(), v.double().cpu().numpy(), [0, 600])
    assert g.map.table[0, :5].tolist() == list(range(n_pages - 8, n_pages - 3))
    a, b = g.gather(n_rows=600, cu_rows=ints([0, 600]), dtype=F32)
    np.testing.assert_array_equal(a.double().cpu().numpy(), r.kv(0)[0])
    np.testing.assert_array_equal(b.double().cpu().numpy(), r.kv(0)[1])
    q = torch.randn(1, 16, d, device="cuda:0").to(BF)
    o, lse = g.attend(q, return_lse=True)
    check_attention(r, q, [0, 1], 1 / np.sqrt(d), True, o, lse)
    keep = torch.zeros(1, 600, dtype=torch.uint8, device="cuda:0")
    keep[0, ::3] = 1
    g.compact(keep)
    assert g.map.lens.item() == 200 and g.map.table[0, :2].tolist() == [n_pages - 3, n_pages - 2] and g.status() == 0
    a, b = g.gather(n_rows=200, cu_rows=ints([0, 200]), dtype=F32)
    np.testing.assert_array_equal(b.double().cpu().numpy(), r.kv(0)[1][::3])


def test_refusals_of_the_binding(im):
    g = im.KV4Cache(2, 2, 4, 2, 64, 16)
    k = torch.zeros(2, 2, 64, dtype=BF, device="cuda:0")
    ok = ints([0, 1, 2])
    for bad in (lambda: g.append(k.float(), k.float(), ok), lambda: g.append(k, k[:1], ok), lambda: g.append(k, k, ok[:2]),
                lambda: g.append(k, k, ok.long()), lambda: g.append(k.cpu(), k, ok), lambda: g.append(k[:1], k[:1]),
                lambda: g.append(k[:1].expand(2, 2, 64), k, ok), lambda: g.attend(k.float()), lambda: g.attend(k.transpose(0, 1)),
                lambda: g.attend(k, out=torch.zeros(2, 2, 64, device="cuda:0")), lambda: g.gather(ok), lambda: g.gather(),
                lambda: g.gather(ok.long(), ok), lambda: g.fork(ok), lambda: g.compact(k), lambda: g.rows(1, 1), lambda: g.rows(0, 3),
                lambda: g.append(k, k, map=im.KV4Cache(2, 3, 4, 2, 64, 16).map), lambda: im.KV4Map(ok.long(), ok, ok),
                lambda: im.KV4Cache(2, 2, 4, 2, 64, 16, device="cpu")):
        with pytest.raises(ValueError):
            bad()
    for kw in (dict(head_dim=80), dict(page_size=24), dict(n_pages=0)):
        with pytest.raises(im.IndexMemError):
            im.KV4Cache(**{**dict(n_seqs=1, max_pages=1, n_pages=1, n_kv_heads=1, head_dim=64, page_size=16), **kw})
    with pytest.raises(im.IndexMemError):
        g.fork(ints([0, 1]), map=g.map, to=im.KV4Map(g.map.refs, g.map.table, g.map.lens.clone()))
    with pytest.raises(im.IndexMemError):
        g.attend(torch.zeros(2, 3, 64, dtype=BF, device="cuda:0"))                        # 3 query heads on 2 KV heads
