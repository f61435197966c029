"""Argument checks of the im_kv4 entry points: every refusal comes before anything touches a device, so none needs a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def im():
    from paper_2605_25475_b200 import buildlib
    buildlib.build()
    from paper_2605_25475_b200 import binding
    return binding


FAKE = 0x100000  # never dereferenced: the calls are refused


def describe(im, **kw):
    f = dict(pool=FAKE, k_exp=None, v_exp=None, status=FAKE, n_pages=10, page_size=64, n_kv_heads=2, head_dim=128, n_seqs=3, max_pages=4)
    f.update(kw)
    return im.im_kv4(*[f[n] for n, _ in im.im_kv4._fields_])


def maps(im, at=FAKE, step=0x10000):
    return im.im_kv4_map(at, at + step, at + 2 * step)


def ref(x):
    return None if x is None else C.addressof(x)


def append(im, c, a, b, dtype=0, k=FAKE, ks=0, v=FAKE, vs=0, n=3, cu=FAKE, ws=FAKE, nbytes=1 << 30):
    return im._lib.im_kv4_append(ref(c), ref(a), ref(b), dtype, k, ks, v, vs, n, cu, ws, nbytes, None)


def attend(im, c, m, dtype=0, q=FAKE, qs=0, n=3, cu=FAKE, max_q=1, H=4, scale=0.0, causal=1, out=FAKE, f32=0, lse=None, ws=FAKE,
           nbytes=1 << 40):
    return im._lib.im_kv4_attention(ref(c), ref(m), dtype, q, qs, n, cu, max_q, H, scale, causal, out, f32, lse, ws, nbytes, None)


def test_struct_layout(im):
    assert C.sizeof(im.im_kv4) == 56 and im.im_kv4.n_pages.offset == 32 and C.sizeof(im.im_kv4_map) == 24


def test_page_bytes(im):
    assert im.im_kv4_page_bytes(8, 128, 64) == 8 * 4 * 16 * (128 + 16)
    for bad in ((0, 128, 64), (257, 128, 64), (8, 96, 64), (8, 512, 64), (8, 128, 48), (8, 128, 256), (8, 128, 8)):
        assert im.im_kv4_page_bytes(*bad) == 0, bad


@pytest.mark.parametrize("kw", [dict(pool=None), dict(pool=FAKE + 8), dict(status=None), dict(n_pages=0), dict(page_size=20),
                                dict(head_dim=80), dict(n_kv_heads=0), dict(n_seqs=0), dict(n_seqs=65536), dict(max_pages=0),
                                dict(n_pages=1 << 26), dict(max_pages=1 << 26), dict(n_seqs=65535, max_pages=1 << 20)])
def test_bad_descriptions(im, kw):
    c, m = describe(im, **kw), maps(im)
    assert append(im, c, m, m) == im.IM_ERR_ARG and im._lib.im_last_error().decode().startswith("im_kv4_append: ")
    assert attend(im, c, m) == im.IM_ERR_ARG
    assert im._lib.im_kv4_gather(ref(c), ref(m), 3, FAKE, FAKE, 0, FAKE, FAKE, None) == im.IM_ERR_ARG
    other = maps(im, FAKE * 16)
    assert im._lib.im_kv4_fork(ref(c), ref(m), ref(other), FAKE, None) == im.IM_ERR_ARG
    assert im._lib.im_kv4_compact(ref(c), ref(m), ref(m), FAKE, 64, FAKE, 1 << 40, None) == im.IM_ERR_ARG
    for op in range(3):
        assert im._lib.im_kv4_workspace_bytes(ref(c), op, 3, 4) == 0


def test_bad_maps(im):
    c, m = describe(im), maps(im)
    for bad in (None, im.im_kv4_map(None, FAKE, FAKE), im.im_kv4_map(FAKE, None, FAKE), im.im_kv4_map(FAKE, FAKE, None),
                im.im_kv4_map(FAKE + 2, FAKE, FAKE)):
        assert append(im, c, bad, m) == im.IM_ERR_ARG and append(im, c, m, bad) == im.IM_ERR_ARG
        assert attend(im, c, bad) == im.IM_ERR_ARG
    half = im.im_kv4_map(m.refs, m.table + 16, m.lens)   # a table that overlaps, shifted by a row
    assert append(im, c, m, half) == im.IM_ERR_ARG and "overlap" in im._lib.im_last_error().decode()
    assert im._lib.im_kv4_compact(ref(c), ref(m), ref(half), FAKE, 64, FAKE, 1 << 40, None) == im.IM_ERR_ARG
    assert im._lib.im_kv4_fork(ref(c), ref(m), ref(m), FAKE, None) == im.IM_ERR_ARG  # rows may change places: not in place
    assert im._lib.im_kv4_fork(ref(c), ref(m), ref(maps(im, FAKE * 16)), None, None) == im.IM_ERR_ARG


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dtype=-1), dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2),
                                dict(ks=255), dict(ks=248), dict(vs=260), dict(n=-1), dict(cu=None, n=4)])
def test_append_refusals(im, kw):
    c, m = describe(im), maps(im)
    assert append(im, c, m, m, **kw) == im.IM_ERR_ARG


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(q=None), dict(q=FAKE + 8), dict(out=None), dict(out=FAKE + 4), dict(lse=FAKE + 1),
                                dict(qs=504), dict(qs=516), dict(n=-1), dict(cu=None, n=2), dict(H=0), dict(H=5), dict(H=65536), dict(max_q=-1),
                                dict(scale=-0.5), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_attention_refusals(im, kw):
    c, m = describe(im), maps(im)
    assert attend(im, c, m, **kw) == im.IM_ERR_ARG


def test_workspaces(im):
    c, m = describe(im), maps(im)
    for op, call in ((0, lambda **k: append(im, c, m, m, **k)), (1, lambda **k: attend(im, c, m, **k))):
        need = im._lib.im_kv4_workspace_bytes(ref(c), op, 3, 4)
        assert need > 0 and need % 256 == 0
        for bad in (dict(nbytes=need - 1), dict(ws=None), dict(ws=FAKE + 128)):
            assert call(**bad) == im.IM_ERR_CAPACITY
    need = im._lib.im_kv4_workspace_bytes(ref(c), 2, 200, 0)
    assert need >= 4 * 3 * 200
    assert im._lib.im_kv4_compact(ref(c), ref(m), ref(m), FAKE, 200, FAKE, need - 1, None) == im.IM_ERR_CAPACITY
    assert im._lib.im_kv4_compact(ref(c), ref(m), ref(m), FAKE, 0, FAKE, 1 << 30, None) == im.IM_ERR_ARG
    assert im._lib.im_kv4_compact(ref(c), ref(m), ref(m), None, 200, FAKE, 1 << 30, None) == im.IM_ERR_ARG
    for bad in ((3, 1, 1), (-1, 1, 1), (0, -1, 1), (1, 1, 0), (1, 1, 3)):
        assert im._lib.im_kv4_workspace_bytes(ref(c), *bad) == 0


def test_gather_refusals(im):
    c, m = describe(im), maps(im)
    g = lambda n=3, cu=FAKE, dt=0, k=FAKE, v=FAKE: im._lib.im_kv4_gather(ref(c), ref(m), n, cu, FAKE, dt, k, v, None)  # noqa: E731
    for kw in (dict(n=-1), dict(cu=None, n=5), dict(dt=3), dict(k=None, v=None), dict(k=FAKE + 8), dict(v=FAKE + 8)):
        assert g(**kw) == im.IM_ERR_ARG
    assert g(n=0, k=None, v=None) == im.IM_OK  # nothing to read


@pytest.mark.parametrize("page_size", [16, 128])
def test_lengths_leave_room_to_be_rounded_up(im, page_size):
    """Kernels round a length up to their tiles in 32 bits: the last 2^16 lengths below 2^31 are refused."""
    most = (2 ** 31 - 2 ** 16) // page_size
    kw = dict(page_size=page_size, n_seqs=1, n_kv_heads=1)
    for name in ("max_pages", "n_pages"):
        for op in (0, 1, 2):
            assert im._lib.im_kv4_workspace_bytes(ref(describe(im, **kw, **{name: most})), op, 1, 1) > 0
            assert im._lib.im_kv4_workspace_bytes(ref(describe(im, **kw, **{name: most + 1})), op, 1, 1) == 0
