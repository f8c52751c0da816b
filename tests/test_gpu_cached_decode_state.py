"""The decode loop's own state (paper_2607_02119_amd/cached_decode.py): what it reports, how large
its steps may be, and that every row's cache holds what was appended for it."""
import numpy as np
import pytest

import _cache_ref as ref
import test_gpu_cache as base

torch = pytest.importorskip("torch")
mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


def test_status_of_a_workspace_that_was_replaced():
    """A bit that a step set before the workspace grew is still reported, once."""
    from paper_2607_02119_amd.cached_decode import CachedDecode
    loop = CachedDecode(rows=4, bound=100, keep=70, recent=20, Hq=4, Hkv=2, D=64, K=3, V=64,
                        V_text=128, seed=3)
    before = loop.workspace
    before[0] = mcd.MCD_DEV_BAD_PAGE
    loop.step()
    assert loop.workspace is not before
    assert loop.status() == mcd.MCD_DEV_BAD_PAGE
    assert loop.status() == 0


def test_more_prompt_tokens_than_a_small_loop_has():
    """800 rows plan up to 6400 tokens in a step."""
    from paper_2607_02119_amd.cached_decode import CachedDecode
    loop = CachedDecode(rows=800, bound=64, keep=40, recent=8, Hq=1, Hkv=1, D=64, K=2, V=32,
                        V_text=64, seed=1)
    seen = []
    loop.step(check=lambda self, b, context, q, out: seen.append(int(b["row_tokens"].sum())))
    assert seen[0] > 4096 and loop.status() == 0


def test_every_row_holds_what_was_appended_for_it(monkeypatch):
    """A mirror of every slot, from the scheduler's plans and the calls' inputs alone: each token's
    keys and values at its position as the append left them, a joining Companion's taken over from
    the Main row of its own request, the positions kept by an eviction, and the received weight
    added up in 64 bits.  Pages, kept positions and weights of the loop against it."""
    from paper_2607_02119_amd.cached_decode import CachedDecode
    H, Hq, D = 2, 4, 64
    loop = CachedDecode(rows=12, bound=100, keep=70, recent=20, Hq=Hq, Hkv=H, D=D, K=3, V=64,
                        V_text=128, seed=5)
    empty = (np.zeros((H, 0, D)), np.zeros((H, 0, D)), np.zeros((H, 0)))
    mirror = {s: empty for s in range(loop.rows)}
    count = dict(copied=0, evicted=0, appended=0)
    state = {}

    plan, move = loop.sched.plan, loop.move

    def planned():
        b = state["plan"] = plan()
        state["joins"] = {}
        for slot, context in zip(b["row_slot"], b["row_context"]):
            if context == 0:
                mirror[int(slot)] = empty
        for head, i in enumerate(b["head_row"]):
            if b["row_kind"][head] == mcd.MCD_ROW_UNCOND and b["step"][head] == 0 and \
                    b["row_context"][i] > loop.null_prompt:
                same = (b["row_req"] == b["row_req"][i]) & (b["row_member"] == 0)
                assert same.sum() == 1
                state["joins"][int(b["row_slot"][i])] = int(b["row_slot"][same][0])
        return b

    def moved(src, dst, keep, recent):
        before = {int(s): mirror[int(s)] for s in src}
        weight = loop.cache.weight.cpu().numpy()
        kept = move(src, dst, keep, recent).cpu().numpy()
        for r, (s, d) in enumerate(zip(src, dst)):
            s, d = int(s), int(d)
            k, v, w = before[s]
            n = w.shape[1]
            if s != d:
                assert state["joins"].pop(d) == s and n <= keep
                count["copied"] += 1
            else:
                assert n > loop.bound and (keep, recent) == (loop.keep, loop.recent)
                count["evicted"] += 1
            m = min(n, keep)
            assert (kept[r, :, m:] == -1).all()
            want = [ref.evict(weight[s, h, :n], keep, recent) for h in range(H)]
            assert all(np.array_equal(kept[r, h, :m], want[h]) for h in range(H))
            mirror[d] = tuple(np.stack([x[h][want[h]] for h in range(H)]) for x in (k, v, w))
        return kept

    append, attend = mcd.mcd_cache_append, mcd.mcd_cache_attend

    def appended(cache, rows, k, v, ws):
        assert not state["joins"]
        append(cache, rows, k, v, ws)
        kr, vr = torch.zeros_like(k, dtype=torch.float32), torch.zeros_like(v, dtype=torch.float32)
        mcd.mcd_cache_read(cache, rows, kr, vr, ws)
        k, v, kr, vr = (x.double().cpu().numpy() for x in (k, v, kr, vr))
        # a key is off by a scale at most, and 3.5 scales are below its block's largest; a
        # value's scale is a sixth of its token's largest, rounded to 8 bits
        top = np.abs(k).reshape(*k.shape[:2], -1, 32).max(-1).repeat(32, -1)
        assert (np.abs(kr - k) <= top / 3.5).all()
        assert (np.abs(vr - v) <= np.abs(v).max(-1, keepdims=True) / 6 * (1 + 2.0 ** -8)).all()
        start = rows.start.cpu().numpy()
        for r, (s, c) in enumerate(zip(rows.slot.cpu().tolist(), rows.context.cpu().tolist())):
            part = slice(start[r], start[r + 1])
            km, vm, w = mirror[s]
            n = start[r + 1] - start[r]
            assert w.shape[1] == c and n == state["plan"]["row_tokens"][r] and \
                s == state["plan"]["row_slot"][r]
            mirror[s] = (np.concatenate([km, kr[part].transpose(1, 0, 2)], 1),
                         np.concatenate([vm, vr[part].transpose(1, 0, 2)], 1),
                         np.concatenate([w, np.zeros((H, n))], 1))
            count["appended"] += n

    def attended(cache, rows, q, out, ws, **kw):
        attend(cache, rows, q, out, ws, **kw)
        start, q = rows.start.cpu().numpy(), q.double().cpu().numpy()
        weight = cache.weight.double().cpu().numpy()
        for r, (s, c) in enumerate(zip(rows.slot.cpu().tolist(), rows.context.cpu().tolist())):
            k, v, w = mirror[s]
            part = q[start[r]:start[r + 1]]
            _, _, add, size = ref.attend(k, v, part, c, D ** -0.5)
            _, tol, _ = base.bounds(k, part, D ** -0.5, torch.bfloat16, add, size)
            got = weight[s, :, :w.shape[1]]
            assert (np.abs(got - (w + add)) <= tol + 2.0 ** -23 * (w + add)).all()
            mirror[s] = (k, v, got)

    monkeypatch.setattr(loop.sched, "plan", planned)
    monkeypatch.setattr(loop, "move", moved)
    monkeypatch.setattr(mcd, "mcd_cache_append", appended)
    monkeypatch.setattr(mcd, "mcd_cache_attend", attended)
    for step in range(120):
        loop.step()
        if step % 6 == 5:
            pages = loop.cache.pages.cpu().numpy()
            weight = loop.cache.weight.cpu().numpy()
            for s, (k, v, w) in mirror.items():
                L = w.shape[1]
                assert L == loop.pool.length[s]
                if L:
                    kd, vd = base.slot_kv(pages, loop.pool.table, s, L, D)
                    assert np.array_equal(kd, k) and np.array_equal(vd, v)
                    assert np.array_equal(weight[s, :, :L], w.astype(np.float32))
    assert count["copied"] > 2 and count["evicted"] > 5 and count["appended"] > 2000
    assert loop.copied == count["copied"] and loop.evicted == count["evicted"]
    assert loop.status() == 0
