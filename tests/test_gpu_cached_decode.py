"""The cache, the scheduler and the head in one loop (paper_2607_02119_amd/cached_decode.py):
attention outputs against the pages' values in 64 bits while rows join, grow, are copied and are
evicted, and the page bookkeeping's invariants."""
import numpy as np
import pytest

import _cache_ref as ref

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


def test_loop_of_scheduler_cache_and_head():
    from paper_2607_02119_amd.cached_decode import CachedDecode
    loop = CachedDecode(rows=12, bound=100, keep=70, recent=20, Hq=4, Hkv=2, D=64, K=3, V=64,
                        V_text=128, seed=3)
    checked = 0

    def check(loop, b, context, q, out):
        nonlocal checked
        pages = loop.cache.pages.cpu().numpy()
        start = np.concatenate([[0], np.cumsum(b["row_tokens"])])
        for i in (0, len(context) - 1):
            n, slot = int(b["row_tokens"][i]), int(b["row_slot"][i])
            L = int(context[i]) + n
            k, v = ref.decode_pages(pages[loop.pool.table[slot, :-(-L // 64)]], 64)
            k, v = (x.transpose(1, 0, 2, 3).reshape(2, -1, 64)[:, :L] for x in (k, v))
            part = slice(start[i], start[i] + n)
            o, _, _, size = ref.attend(k, v, q[part].double().cpu().numpy(), int(context[i]),
                                       0.125)
            got = out[part].double().cpu().numpy()
            # the output's rounding to bf16 (2^-8), fp32 sums below
            assert (np.abs(got - o) <= (2.0 ** -8 + 2.0 ** -13) * size + 1e-30).all()
            checked += 1

    decoded = 0
    for step in range(160):
        decoded += loop.step(check if step % 8 == 7 else None)
        held = sorted(p for pages in loop.pool.pages for p in pages)
        assert len(set(held)) == len(held)                        # no page has two owners
        assert len(held) + len(loop.pool.free) == loop.cache.pages.shape[0]
        assert (loop.pool.length <= loop.bound).all() and (loop.tokens >= 0).all() \
            if decoded else True
    assert checked >= 30 and loop.evicted > 5 and loop.copied > 2
    assert loop.status() == 0
