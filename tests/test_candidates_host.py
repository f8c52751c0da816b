"""Page tables and log probabilities without a GPU: what the library refuses before any launch."""
import ctypes

import numpy as np
import pytest

mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")
torch = pytest.importorskip("torch")

FAKE = 0x100000   # never dereferenced: refused before any launch


def _pages(**kw):
    a = dict(n_slots=4, max_pages=8, n_pages=50, table=FAKE, refs=FAKE + 0x1000)
    a.update(kw)
    return mcd.mcd_cache_pages(**a)


BAD_PAGES = [dict(n_slots=0), dict(max_pages=0), dict(n_pages=0), dict(table=None), dict(refs=None),
             dict(table=FAKE + 2), dict(refs=FAKE + 0x1001), dict(max_pages=1 << 25),
             dict(n_slots=1 << 30, max_pages=1 << 20), dict(refs=FAKE + 64)]


def _reserve(p=None, **kw):
    a = dict(R=3, n_tokens=9, max_tokens=5, max_context=500, slot=FAKE + 0x2000,
             context=FAKE + 0x3000, tokens=FAKE + 0x4000, start=FAKE + 0x5000, where=FAKE + 0x6000,
             row=FAKE + 0x7000, position=FAKE + 0x8000, workspace=FAKE, workspace_bytes=1 << 20)
    a.update(kw)
    return mcd._mcd_cache_reserve(ctypes.byref(p or _pages()),
                                  ctypes.byref(mcd.mcd_cache_reserve_args(**a)), None)


def _calls(p, R=3, slot=FAKE + 0x2000, length=FAKE + 0x3000, ws=FAKE, wb=256):
    ref = ctypes.byref(p)
    return [mcd._mcd_cache_release(ref, R, slot, length, ws, wb, None),
            mcd._mcd_cache_share(ref, R, slot, FAKE + 0x4000, length, ws, wb, None)]


def test_page_calls_refuse():
    for b in BAD_PAGES:
        p = _pages(**b)
        assert _calls(p) == [mcd.MCD_E_INVALID] * 2, b
        assert _reserve(p) == mcd.MCD_E_INVALID, b
        assert mcd._mcd_cache_count(ctypes.byref(p), FAKE, 256, None) == mcd.MCD_E_INVALID, b
        assert mcd._mcd_cache_pages_workspace_bytes(ctypes.byref(p), 3) == 0
    p = _pages()
    for b in (dict(R=-1), dict(R=65536), dict(slot=FAKE + 0x2002), dict(length=FAKE + 0x1004),
              dict(slot=FAKE + 4 * 31), dict(ws=None), dict(ws=FAKE + 128)):
        assert _calls(p, **b) == [mcd.MCD_E_INVALID] * 2, b
    assert _calls(p, wb=255) == [mcd.MCD_E_WORKSPACE] * 2
    assert mcd._mcd_cache_count(ctypes.byref(p), FAKE, 255, None) == mcd.MCD_E_WORKSPACE
    assert mcd._mcd_cache_share(ctypes.byref(p), 3, None, None, FAKE, FAKE, 256, None) \
        == mcd.MCD_E_INVALID
    assert _calls(p, R=0, ws=None) == [mcd.MCD_OK] * 2


def test_reserve_refuses():
    for b in (dict(R=-1), dict(R=65536), dict(n_tokens=-1), dict(max_tokens=-1), dict(max_tokens=10),
              dict(max_context=-1), dict(max_context=(1 << 30) + 1), dict(context=None),
              dict(tokens=None), dict(start=None), dict(where=FAKE + 0x6004), dict(row=FAKE + 0x7002),
              dict(position=FAKE + 0x8001), dict(start=FAKE + 0x3008), dict(start=FAKE + 0x4000),
              dict(start=FAKE + 0x2000), dict(where=FAKE + 0x5008), dict(row=FAKE + 0x8000),
              dict(position=FAKE + 0x1000), dict(row=FAKE + 8), dict(where=FAKE + 0x3000),
              dict(context=FAKE + 4), dict(workspace=None), dict(workspace=FAKE + 64),
              dict(R=0, n_tokens=9)):
        assert _reserve(**b) == mcd.MCD_E_INVALID, b
    need = mcd._mcd_cache_pages_workspace_bytes(ctypes.byref(_pages()), 3)
    assert need > 256 and _reserve(workspace_bytes=need - 1) == mcd.MCD_E_WORKSPACE
    assert _reserve(R=0, n_tokens=0, max_tokens=0, workspace=None) == mcd.MCD_OK
    assert mcd._mcd_cache_reserve(ctypes.byref(_pages()), None, None) == mcd.MCD_E_INVALID
    # a workspace serves fewer rows
    sizes = [mcd._mcd_cache_pages_workspace_bytes(ctypes.byref(_pages()), R) for R in range(300)]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_page_tensors_are_checked():
    with pytest.raises(ValueError):
        mcd.CachePages(torch.zeros((3, 4), dtype=torch.int64), 5)
    pages = mcd.CachePages(torch.zeros((3, 4), dtype=torch.int32), 5)
    ws, i = torch.zeros(4096, dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):                  # not on the GPU
        mcd.mcd_cache_release(pages, i, ws)
    with pytest.raises(ValueError):
        mcd.mcd_cache_release(pages, i, ws, length=i[:2])
    with pytest.raises(ValueError):
        mcd.mcd_cache_share(pages, i, i.long(), i, ws)
    with pytest.raises(ValueError):
        mcd.mcd_cache_reserve(pages, i, i, i, ws)     # start of R


def _logprobs(**kw):
    a = dict(n=4, K=2, V=100, T=3, pad_id=100, dtype=mcd.MCD_F32, logits=FAKE, logits_stride=200,
             V_stream=None, token_rows=4, tokens=FAKE + 0x10000, token_row=None,
             logprob=FAKE + 0x20000, entropy=FAKE + 0x30000, top_ids=FAKE + 0x40000,
             top_logprobs=FAKE + 0x50000, workspace=FAKE + 0x60000, workspace_bytes=1 << 20)
    a.update(kw)
    return mcd._mcd_logprobs(ctypes.byref(mcd.mcd_logprobs_args(**a)), None)


def test_logprobs_refuse():
    streams = np.array([100, 101], np.int32)
    none = np.array([100, 0], np.int32)
    for b in (dict(n=-1), dict(K=0), dict(K=33), dict(V=0), dict(T=-1), dict(pad_id=0),
              dict(pad_id=99), dict(dtype=5), dict(logits=None), dict(tokens=None),
              dict(logprob=None), dict(logits_stride=199), dict(token_rows=3), dict(token_rows=0),
              dict(T=0), dict(top_ids=None, top_logprobs=None), dict(logits=FAKE + 2),
              dict(logits=FAKE + 1, dtype=mcd.MCD_BF16), dict(tokens=FAKE + 0x10002),
              dict(entropy=FAKE + 0x30001), dict(V_stream=streams.ctypes.data),
              dict(V_stream=none.ctypes.data), dict(entropy=FAKE + 0x20004),
              dict(logprob=FAKE + 0x10010), dict(top_ids=FAKE + 400), dict(top_ids=FAKE + 0x50020),
              dict(token_row=FAKE + 0x20000), dict(workspace=None), dict(workspace=FAKE + 0x60080),
              dict(n=1 << 30, K=4, token_rows=1 << 30)):
        assert _logprobs(**b) == mcd.MCD_E_INVALID, b
    for b in (dict(T=33), dict(V=(1 << 19) + 1, logits_stride=1 << 21, pad_id=-1)):
        assert _logprobs(**b) == mcd.MCD_E_UNSUPPORTED, b
    assert _logprobs(workspace_bytes=255) == mcd.MCD_E_WORKSPACE
    assert _logprobs(V=5000, pad_id=-1, logits_stride=10000, logits=FAKE << 4, workspace_bytes=256) \
        == mcd.MCD_E_WORKSPACE
    assert _logprobs(n=0, logits=None, workspace=None) == mcd.MCD_OK
    assert mcd._mcd_logprobs(None, None) == mcd.MCD_E_INVALID


def test_logprobs_workspace_serves_smaller_calls():
    f = mcd._mcd_logprobs_workspace_bytes
    for n in (1, 7, 64):
        for V in (1, 4096, 4097, 8193, 200000, 1 << 19):
            for T in (0, 1, 32):
                most = f(n, 4, V, T)
                assert most >= 256
                assert f(n // 2, 4, V, T) <= most and f(n, 3, V, T) <= most
                assert f(n, 4, V // 2 + 1, T) <= most and f(n, 4, V, T // 2) <= most
    assert f(1, 1, 0, 0) == f(1, 0, 1, 0) == f(-1, 1, 1, 0) == f(1, 1, 1, 33) == 0


def test_logprob_tensors_are_checked():
    x, i, f = torch.zeros(4, 2, 10), torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, 2)
    ws = torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(ValueError, match="not on the GPU"):
        mcd.mcd_logprobs(x, i, f, ws)
    for a, kw in (((x.double(), i, f), {}), ((x[0], i, f), {}), ((x.transpose(1, 2), i, f), {}),
                  ((x, i.long(), f), {}), ((x, i, f[:3]), {}), ((x, i, f.half()), {}),
                  ((x, i, f), dict(entropy=f[:, :1])), ((x, i, f), dict(top_ids=i)),
                  ((x, i, f), dict(token_row=i[:, 0])),
                  ((x.flatten(1), i, f), dict(V_stream=[10, 11]))):
        with pytest.raises(ValueError):
            mcd.mcd_logprobs(*a, ws, **kw)


def test_logprobs_of_more_vectors_than_a_launch_takes():
    """A launch has fewer than 2^32 threads: 2^24 workgroups of 256, each for a vector's part of up to
    8192 logits or for four vectors of up to 1024."""
    f = mcd._mcd_logprobs_workspace_bytes
    for V, most in ((1, (1 << 26) - 4), (1024, (1 << 26) - 4), (1025, (1 << 24) - 1),
                    (4096, (1 << 24) - 1), (8192, (1 << 24) - 1), (8193, (1 << 23) - 1),
                    (151936, ((1 << 24) - 1) // 19), (1 << 19, ((1 << 24) - 1) // 64)):
        for T in (0, 1, 5):
            assert f(most, 1, V, T) > 0 and f(most // 16, 16, V, T) > 0
            assert f(most + 1, 1, V, T) == 0 and f(most // 16 + 1, 16, V, T) == 0
        b = dict(n=most + 1, K=1, V=V, T=0, pad_id=-1, logits=1 << 60, logits_stride=V,
                 token_rows=most + 1, token_row=None, entropy=None, top_ids=None,
                 top_logprobs=None, workspace_bytes=1 << 50)
        assert _logprobs(**b) == mcd.MCD_E_UNSUPPORTED, V


def test_attention_of_more_tiles_than_a_launch_takes():
    """65535 rows of 257 heads and prompts of 2^26 tokens: more than 2^24 - 1 workgroups.  Together
    four single rows are a workgroup's, so of rows that share pages only the prompts are refused."""
    route = mcd._lib.mcd_cache_attend_route
    route.restype = ctypes.c_int
    for Hkv, D, rows in ((257, 64, dict(R=65535, n_tokens=65535, max_tokens=1, max_context=5000)),
                         (16, 256, dict(R=1, n_tokens=1 << 26, max_tokens=1 << 26,
                                        max_context=1 << 26, start=FAKE))):
        cache = mcd.mcd_cache(Hkv=Hkv, D=D, n_slots=70000, max_pages=1 << 20, n_pages=9, pages=FAKE,
                              table=FAKE)
        r = mcd.mcd_cache_rows(slot=None, context=FAKE, **rows)
        a = mcd.mcd_cache_attend_args(Hq=Hkv, dtype=mcd.MCD_BF16, scale=0.1, q=FAKE,
                                      q_stride=Hkv * D, out=1 << 60, out_stride=Hkv * D,
                                      workspace=FAKE, workspace_bytes=1 << 50)
        ref = [ctypes.byref(x) for x in (cache, r, a)]
        assert mcd._mcd_cache_attend(*ref, None) == mcd.MCD_E_INVALID
        assert "too many query rows" in mcd.mcd_last_error()
    g = mcd.mcd_cache_groups(n=1, max_rows=65535, max_prefix=4096, max_own=1 << 26, start=FAKE,
                             prefix=FAKE)
    for way in (-1, 0, 1):
        assert route(*ref[:2], ctypes.byref(g), ref[2], way, None) == mcd.MCD_E_INVALID
        assert "too many query rows" in mcd.mcd_last_error()
