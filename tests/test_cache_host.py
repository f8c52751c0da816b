"""The 4-bit key/value cache without a GPU: its reference against itself and closed forms, and
what the library refuses before any launch."""
import ctypes

import numpy as np
import pytest

import _cache_ref as ref

mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")
torch = pytest.importorskip("torch")

FAKE = 0x10000   # never dereferenced: refused before any launch


@pytest.mark.parametrize("D", [64, 128, 256])
def test_page_layout_is_a_permutation(D):
    """Every code of a page has a nibble of its own, and the page is its codes and scales."""
    keys = {t * D + c for t in range(64) for c in range(D)}
    values = {ref.value_nibble(D, t, c) for t in range(64) for c in range(D)}
    assert keys == set(range(64 * D)) and values == set(range(64 * D, 128 * D))
    assert mcd.mcd_cache_page_bytes(D) == ref.page_bytes(D) == 66 * D + 128
    assert mcd.mcd_cache_page_bytes(D + 32) == 0


@pytest.mark.parametrize("D", [64, 128, 256])
def test_reference_round_trip(D):
    rng = np.random.default_rng(D)
    page = np.zeros(ref.page_bytes(D), np.uint8)
    k = rng.standard_normal((64, D)).astype(np.float32)
    v = rng.standard_normal((64, D)).astype(np.float32)
    for t in rng.permutation(64):
        ref.put(page, D, t, k[t], v[t])
    dk, dv = ref.decode_pages(page[None, None], D)
    for t in (0, 15, 16, 33, 63):
        one = ref.get(page, D, t)
        assert np.array_equal(one[0], dk[0, 0, t]) and np.array_equal(one[1], dv[0, 0, t])
    # no key is further off than half the widest step (between 4 and 6) of its scale
    for t in range(64):
        for b in range(D // 32):
            block = k[t, 32 * b:32 * b + 32]
            s = 2.0 ** (ref.key_exponent(block) - 127)
            assert np.abs(dk[0, 0, t, 32 * b:32 * b + 32] - block).max() <= s
            assert 3.5 * s < np.abs(block).max() <= 7 * s
        s = ref.value_scale(v[t])
        assert np.abs(dv[0, 0, t] - v[t]).max() <= s


def test_reference_codes_and_scales():
    """Levels map to themselves, midpoints to the even code, and larger values to the largest."""
    for c, x in enumerate(ref.LEVELS):
        assert ref.code(x, 1.0) == c and ref.code(-x, 1.0) == c + 8
    mid = (ref.LEVELS[1:] + ref.LEVELS[:-1]) / 2
    assert [ref.code(x, 1.0) for x in mid] == [0, 2, 2, 4, 4, 6, 6]
    assert ref.code(100.0, 1.0) == 7
    assert ref.key_exponent(np.array([7.0])) == 127 and ref.key_exponent(np.array([7.01])) == 128
    assert ref.key_exponent(np.zeros(32)) == 1 and ref.key_exponent(np.array([np.inf])) == 255
    assert ref.value_scale(np.array([6.0, -3.0])) == 1.0


def test_reference_eviction():
    assert ref.evict(np.array([1.0, 5, 5, 0, 2]), 3, 1).tolist() == [1, 2, 4]
    assert ref.evict(np.array([3.0, 3, 3, 3, 9]), 3, 1).tolist() == [0, 1, 4]
    assert ref.evict(np.array([np.nan, -np.inf, 0, 1]), 2, 0).tolist() == [2, 3]
    assert ref.evict(np.array([np.nan, -np.inf, 0, 1]), 3, 0).tolist() == [1, 2, 3]
    assert ref.evict(np.array([1.0, 2]), 5, 0).tolist() == [0, 1]


# ---- refusals ----------------------------------------------------------------

def _cache(**kw):
    a = dict(Hkv=2, D=128, n_slots=3, max_pages=4, n_pages=9, pages=FAKE, table=FAKE, weight=FAKE)
    a.update(kw)
    return mcd.mcd_cache(**a)


def _rows(**kw):
    a = dict(R=3, n_tokens=3, max_tokens=1, max_context=100, slot=None, context=FAKE, start=None)
    a.update(kw)
    return mcd.mcd_cache_rows(**a)


def _move(f, c=None, r=None, dtype=mcd.MCD_BF16, k=FAKE, ks=256, v=FAKE, vs=256, ws=FAKE, wb=256):
    c, r = c or _cache(), r or _rows()
    return f(ctypes.byref(c), ctypes.byref(r), dtype, k, ks, v, vs, ws, wb, None)


BAD_CACHES = [dict(Hkv=0), dict(n_slots=0), dict(max_pages=0), dict(n_pages=0), dict(pages=None),
              dict(table=None), dict(pages=FAKE + 8), dict(max_pages=1 << 26)]
BAD_ROWS = [dict(R=-1), dict(n_tokens=-1), dict(max_tokens=2), dict(max_context=-1),
            dict(context=None), dict(n_tokens=4), dict(R=70000, n_tokens=70000),
            dict(start=FAKE, max_tokens=0), dict(start=FAKE, max_tokens=4)]


@pytest.mark.parametrize("name", ["append", "read"])
def test_append_and_read_refuse(name):
    f = getattr(mcd, f"_mcd_cache_{name}")
    for b in BAD_CACHES:
        assert _move(f, c=_cache(**b)) == mcd.MCD_E_INVALID, b
    for b in BAD_ROWS:
        assert _move(f, r=_rows(**b)) == mcd.MCD_E_INVALID, b
    for D in (0, 32, 96, 512):
        assert _move(f, c=_cache(D=D)) == mcd.MCD_E_UNSUPPORTED
    for b in (dict(dtype=7), dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(vs=255),
              dict(ks=260), dict(ks=128), dict(ws=None), dict(ws=FAKE + 128)):
        assert _move(f, **b) == mcd.MCD_E_INVALID, b
    assert _move(f, wb=128) == mcd.MCD_E_WORKSPACE
    assert f(None, ctypes.byref(_rows()), 1, FAKE, 256, FAKE, 256, FAKE, 256, None) \
        == mcd.MCD_E_INVALID
    assert "null cache" in mcd.mcd_last_error()
    # nothing to do is not an error, whatever the buffers
    assert _move(f, r=_rows(R=0, n_tokens=0, max_tokens=0, start=FAKE), k=None, v=None) == mcd.MCD_OK


def _attend(c=None, r=None, **kw):
    a = dict(Hq=4, dtype=mcd.MCD_BF16, scale=0.1, q=FAKE, q_stride=512, out=FAKE, out_stride=512,
             lse=None, weight_out=None, workspace=FAKE, workspace_bytes=1 << 30)
    a.update(kw)
    c, r = c or _cache(), r or _rows()
    return mcd._mcd_cache_attend(ctypes.byref(c), ctypes.byref(r),
                                 ctypes.byref(mcd.mcd_cache_attend_args(**a)), None)


def test_attend_refuses():
    for b in BAD_CACHES:
        assert _attend(c=_cache(**b)) == mcd.MCD_E_INVALID, b
    for b in BAD_ROWS:
        assert _attend(r=_rows(**b)) == mcd.MCD_E_INVALID, b
    for b in (dict(Hq=3), dict(Hq=0), dict(dtype=9), dict(scale=0.0), dict(scale=-1.0),
              dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None),
              dict(q=FAKE + 2), dict(q_stride=500), dict(out_stride=516), dict(workspace=None)):
        assert _attend(**b) == mcd.MCD_E_INVALID, b
    assert _attend(workspace_bytes=256) == mcd.MCD_E_WORKSPACE
    assert mcd._mcd_cache_attend(ctypes.byref(_cache()), ctypes.byref(_rows()), None, None) \
        == mcd.MCD_E_INVALID
    n = mcd._mcd_cache_workspace_bytes
    assert n(ctypes.byref(_cache()), ctypes.byref(_rows()), 4) >= 256
    assert n(ctypes.byref(_cache()), ctypes.byref(_rows()), 3) == 0
    assert n(ctypes.byref(_cache(D=96)), ctypes.byref(_rows()), 4) == 0


def _evict(c=None, d=None, **kw):
    a = dict(R=3, max_length=200, keep=64, recent=8, slot=None, length=FAKE, kept=FAKE,
             length_out=FAKE, workspace=FAKE, workspace_bytes=256)
    a.update(kw)
    c, d = c or _cache(), d or _cache()
    return mcd._mcd_cache_evict(ctypes.byref(c), ctypes.byref(d),
                                ctypes.byref(mcd.mcd_cache_evict_args(**a)), None)


def test_evict_refuses():
    for b in BAD_CACHES:
        assert _evict(c=_cache(**b)) == mcd.MCD_E_INVALID, b
        assert _evict(d=_cache(**b)) == mcd.MCD_E_INVALID, b
    for b in (dict(R=-1), dict(R=4), dict(keep=0), dict(recent=-1), dict(recent=65),
              dict(max_length=-1), dict(length=None), dict(kept=None), dict(length_out=None),
              dict(workspace=FAKE + 4)):
        assert _evict(**b) == mcd.MCD_E_INVALID, b
    assert _evict(workspace_bytes=0) == mcd.MCD_E_WORKSPACE
    assert _evict(c=_cache(weight=None)) == mcd.MCD_E_INVALID
    assert _evict(d=_cache(Hkv=1)) == mcd.MCD_E_INVALID
    assert _evict(d=_cache(D=64)) == mcd.MCD_E_INVALID
    assert _evict(R=0, length=None) == mcd.MCD_OK


def test_binding_refuses_what_the_library_cannot_see():
    """Types, shapes and strides are known to the binding only."""
    cache = mcd.Cache.alloc(4, 2, 64, 2, 3, weights=True, device="cpu")
    rows = mcd.CacheRows(torch.zeros(2, dtype=torch.int32), max_context=10)
    k = torch.zeros((2, 2, 64))
    ws = torch.zeros(256, dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    bad = [k[:1], k[:, :1], torch.zeros((2, 2, 128)), k.double(), k.transpose(0, 1)[:, :, ::2],
           torch.zeros((2, 64, 2)).transpose(1, 2), torch.zeros((2, 4, 64))[:, ::2]]
    for b in bad:
        with pytest.raises(ValueError):
            mcd.mcd_cache_append(cache, rows, b, k, ws)
    with pytest.raises(ValueError):
        mcd.mcd_cache_append(cache, rows, k, k.bfloat16(), ws)
    with pytest.raises(ValueError):
        mcd.mcd_cache_attend(cache, rows, k, k, ws, lse=torch.zeros(3))
    with pytest.raises(ValueError):
        mcd.mcd_cache_attend(cache, rows, k, k, ws, weight_out=torch.zeros(3))
    # host memory: the kernels would fault on it
    for call in (lambda: mcd.mcd_cache_append(cache, rows, k, k, ws),
                 lambda: mcd.mcd_cache_attend(cache, rows, k, k, ws),
                 lambda: mcd.mcd_cache_evict(cache, cache, i32(2), 8, 2, i32(2, 2, 8), i32(2), ws,
                                             10)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError):
        mcd.Cache(cache.pages[..., 1:], cache.table, 64)
    with pytest.raises(ValueError):
        mcd.Cache(cache.pages, cache.table.long(), 64)
    with pytest.raises(ValueError):
        mcd.Cache(cache.pages, cache.table, 64, weight=torch.zeros((2, 2, 64)))
    with pytest.raises(ValueError):
        mcd.CacheRows(torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        mcd.CacheRows(torch.zeros(2, dtype=torch.int32), start=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="kept"):
        mcd.mcd_cache_evict(cache, cache, i32(2), 8, 2, i32(2, 2, 7), i32(2), ws, 10)


def test_workspace_of_a_larger_step_serves_smaller_ones():
    """No fewer rows, tokens or positions need more: 8 rows are split where 512 are not, and keep
    scores where more than 1 GiB of them are computed again."""
    rng = np.random.default_rng(6)

    def size(cache, b, Hq, start):
        r = _rows(R=b[0], n_tokens=b[1], max_tokens=b[2], max_context=b[3],
                  start=FAKE if start else None)
        return mcd._mcd_cache_workspace_bytes(ctypes.byref(cache), ctypes.byref(r), Hq)

    def log(lo, hi):
        return int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))

    for _ in range(4000):
        Hkv, G = int(rng.choice([1, 2, 8])), int(rng.choice([1, 2, 3, 4, 5, 8, 9, 16, 17, 64, 100]))
        cache = _cache(Hkv=Hkv, D=int(rng.choice([64, 128, 256])), n_slots=512, max_pages=256,
                       weight=FAKE if rng.random() < 0.5 else None)
        R = log(1, 512)
        mt = log(1, 600) if rng.random() < 0.7 else 1
        N = int(rng.integers(mt, R * mt + 1))
        large = (R, N, mt, log(1, 20000))
        whole = size(cache, large, Hkv * G, True)
        assert whole > 0
        for _ in range(3):
            mt2 = int(rng.integers(1, mt + 1))
            R2 = int(rng.integers(1, R + 1))
            N2 = int(rng.integers(mt2, max(mt2, min(N, R2 * mt2)) + 1))
            small = (R2, N2, mt2, int(rng.integers(1, large[3] + 1)))
            assert size(cache, small, Hkv * G, True) <= whole, (Hkv, G, cache.D, large, small)
            if R2 <= N:
                one = (R2, R2, 1, small[3])
                assert size(cache, one, Hkv * G, False) <= whole, (Hkv, G, cache.D, large, one)
    # without weights there is no room for scores
    need = size(_cache(weight=None, n_slots=512, max_pages=256), (512, 512, 1, 16384), 8, True)
    assert need < 1 << 24 < size(_cache(n_slots=512, max_pages=256), (512, 512, 1, 16384), 8, True)


def test_arrays_that_are_not_aligned_to_their_elements():
    for b in (dict(weight=FAKE + 2), dict(table=FAKE + 1)):
        assert _attend(c=_cache(**b)) == mcd.MCD_E_INVALID, b
        assert _move(mcd._mcd_cache_append, c=_cache(**b)) == mcd.MCD_E_INVALID, b
        assert _evict(c=_cache(**b)) == mcd.MCD_E_INVALID, b
    for b in (dict(weight_out=FAKE + 2), dict(lse=FAKE + 3)):
        assert _attend(**b) == mcd.MCD_E_INVALID, b


def test_out_over_the_queries_is_refused():
    """A query row is read before its own output is written, so out may be q; the received weight
    is added up from the queries after that."""
    row = 4 * 128 * 2                                         # bytes of a token
    for out, stride in ((0, 512), (16, 512), (row - 16, 512), (16 - row, 512), (2 * row, 512),
                        (2 * row - 16, 1024), (16, 520), (-2 * row + 16, 512)):
        for q_stride in (512, 520):
            bad = dict(weight_out=FAKE << 8, q=FAKE << 4, out=(FAKE << 4) + out, out_stride=stride,
                       q_stride=q_stride)
            assert _attend(**bad) == mcd.MCD_E_INVALID, (out, stride, q_stride)
            assert "overlap" in mcd.mcd_last_error()
            if out or stride != q_stride:
                assert _attend(**dict(bad, weight_out=None)) == mcd.MCD_E_INVALID


def test_eviction_in_place_is_refused():
    """Every head's workgroup reads a row's length and slot, and one of them writes length_out."""
    at = lambda n: (FAKE << 4) + n  # noqa: E731
    good = dict(length=at(0), slot=at(12), length_out=at(24), kept=at(36))
    for b in (dict(length_out=at(0)), dict(length_out=at(-8)), dict(length_out=at(20)),
              dict(kept=at(8)), dict(kept=at(16)), dict(kept=at(32)), dict(length_out=at(100)),
              dict(kept=at(40 - 3 * 2 * 64 * 4))):
        assert _evict(**dict(good, **b)) == mcd.MCD_E_INVALID, b
        assert "overlap" in mcd.mcd_last_error()


def test_room_for_scores_beyond_64_bits():
    """65531 rows x 65454 heads x 12599637 pages x 1 KiB wrap to 361 MiB in 64 bits: rows within
    these bounds keep scores of up to 1 GiB, and more are not kept."""
    rows = dict(R=65531, n_tokens=1, max_tokens=1, max_context=12599637 * 64, start=FAKE)
    a, b = (mcd._mcd_cache_workspace_bytes(
        ctypes.byref(_cache(Hkv=65454, D=64, n_slots=65531, max_pages=12599637, weight=w)),
        ctypes.byref(_rows(**rows)), 65454) for w in (FAKE, None))
    assert b > 0 and a - b == 1 << 30


def test_weight_out_beside_the_weights_is_refused():
    """In place or apart: shifted, one position's sum would be another's start."""
    size = 3 * 2 * 4 * 64 * 4
    for shift in (4, -4, 256, size - 4, 4 - size):
        at = dict(c=_cache(weight=FAKE << 8), weight_out=(FAKE << 8) + shift, q=FAKE, out=FAKE << 4)
        assert _attend(**at) == mcd.MCD_E_INVALID, shift
        assert "apart" in mcd.mcd_last_error()
        assert _attend(r=_rows(R=3, n_tokens=0, max_tokens=0, start=FAKE), **at) == mcd.MCD_E_INVALID
