"""Several continuations of each prompt, from page tables to log probabilities, as a serving program
runs them: the candidates' pages, appended keys and values, attention over the shared pages, a head
step, the log probabilities of what it drew, the best candidate of each prompt, and all pages back."""
import numpy as np
import pytest

import _cache_ref as ref

torch = pytest.importorskip("torch")
mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")

from test_gpu_cache import bounds, i32, slot_kv  # noqa: E402
from test_gpu_logprobs import reference  # noqa: E402

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

BF16 = torch.bfloat16
HQ, HKV, D, K, V = 8, 2, 64, 3, 200


class Serving:
    """Prompts with candidates; the device keeps tables, contexts and log probabilities."""

    def __init__(self, prompts, candidates, seed=0, steps=6):
        self.rng = np.random.default_rng(seed)
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.lengths = np.array(prompts)
        self.P, self.n = len(prompts), candidates
        self.R = self.P * candidates
        # slots: prompts, then candidates; a page more than a slot's longest sequence
        columns = (max(prompts) + steps) // 64 + 2
        n_pages = sum(-(-p // 64) for p in prompts) + 3 * self.R + 2
        self.cache = mcd.Cache.alloc(n_pages, HKV, D, self.P + self.R, columns)
        self.pages = mcd.CachePages(self.cache.table, n_pages)
        self.ws = self.pages.workspace(self.P + self.R)
        self.kv = [torch.randn((p, 2 * HKV, D), generator=self.gen, device="cuda").to(BF16)
                   for p in prompts]
        self.head = mcd.Head(torch.randn((K, V, HQ * D), generator=self.gen, device="cuda").to(BF16)
                             * 0.02, np.arange(K), V)
        self.of = np.repeat(np.arange(self.P), candidates)
        self.slot = i32(self.P + np.arange(self.R))
        self.shared = self.lengths // 64 * 64
        self.groups = mcd.CacheGroups(i32(np.arange(self.P + 1) * candidates), i32(self.lengths),
                                      candidates, int(self.lengths.max()), 64 + steps)
        self.score = torch.zeros(self.R, dtype=torch.float64, device="cuda")
        self.steps = steps

    def append(self, slot, context, tokens, kv):
        """Pages for the rows' tokens, and their keys and values into them."""
        N = int(np.sum(tokens))
        start = torch.zeros(len(tokens) + 1, dtype=torch.int32, device="cuda")
        where = torch.zeros(N, dtype=torch.int64, device="cuda")
        context = i32(context)
        mcd.mcd_cache_reserve(self.pages, context, i32(tokens), start, self.ws, slot=slot,
                              n_tokens=N, max_tokens=int(np.max(tokens)),
                              max_context=self.cache.max_pages * 64, where=where)
        rows = mcd.CacheRows(context, start=start, slot=slot, n_tokens=N,
                             max_tokens=int(np.max(tokens)), max_context=self.cache.max_pages * 64)
        mcd.mcd_cache_append(self.cache, rows, kv[:, :HKV], kv[:, HKV:], self.ws)
        assert bool((where >= 0).all())
        return rows

    def prefill(self):
        self.append(i32(np.arange(self.P)), np.zeros(self.P), self.lengths, torch.cat(self.kv))

    def fork(self):
        """Every candidate on its prompt's whole pages; the rest of the prompt again, its own."""
        mcd.mcd_cache_share(self.pages, self.slot, i32(self.of), i32(self.lengths[self.of]), self.ws)
        rest = self.lengths - self.shared
        if rest.any():
            self.append(self.slot, self.shared[self.of], rest[self.of],
                        torch.cat([self.kv[p][self.shared[p]:] for p in self.of]))
        mcd.mcd_cache_release(self.pages, i32(np.arange(self.P)), self.ws)   # the prompts' slots go


def test_best_of_n():
    s = Serving([130, 64, 301], 5)
    s.prefill()
    s.fork()
    context = s.lengths[s.of].copy()
    history = []
    for step in range(s.steps):
        qkv = torch.randn((s.R, HQ + 2 * HKV, D), generator=s.gen, device="cuda").to(BF16)
        rows = s.append(s.slot, context, np.ones(s.R, int), qkv[:, HQ:])
        # groups of candidates: pages of a prompt once for its five rows
        ws = s.cache.workspace(rows, HQ, groups=s.groups)
        out = torch.zeros((s.R, HQ, D), dtype=BF16, device="cuda")
        mcd.mcd_cache_attend_shared(s.cache, rows, s.groups, qkv[:, :HQ], out, ws)
        assert mcd.mcd_read_device_status(ws) == 0
        pages, table = s.cache.pages.cpu().numpy(), s.cache.table.cpu().numpy()
        for r in range(s.R):
            k, v = slot_kv(pages, table, s.P + r, context[r] + 1, D)
            q = qkv[r:r + 1, :HQ].double().cpu().numpy()
            scale = float(np.float32(D ** -0.5))
            o, _, w, size = ref.attend(k, v, q, context[r], scale)
            to, _, _ = bounds(k, q, scale, BF16, w, size)
            assert (np.abs(out[r:r + 1].double().cpu().numpy() - o) <= to).all()
        # the head step draws; what it drew, under its scores
        plan = s.head.plan(np.full(s.R, -1, np.int32), np.full(s.R, mcd.MCD_ROW_SOLO, np.uint8))
        full = lambda x, dt: torch.full((s.R,), x, dtype=dt, device="cuda")  # noqa: E731
        tokens = torch.zeros((s.R, K), dtype=torch.int32, device="cuda")
        scores = torch.zeros((s.R, K * V), device="cuda")
        grid = torch.full((s.R, K, 32), -1, dtype=torch.int32, device="cuda")
        mcd.mcd_head_step(
            s.head.handle, R=s.R, counts=plan.counts, plan=plan.dev, hidden=out.view(s.R, HQ * D),
            cfg_w=full(1.0, torch.float32), temperature=full(1.0, torch.float32),
            top_k=full(0, torch.int32), top_p=full(1.0, torch.float32),
            rng_key=torch.arange(s.R, device="cuda"), step=full(step, torch.int32),
            n_frames=full(32, torch.int32), grid_slot=i32(np.arange(s.R)), seed=1,
            tokens_out=tokens, frame_grid=grid, n_slots=s.R, F_max=32, scores=scores,
            workspace=s.head.workspace(s.R))
        lp, H = (torch.zeros((s.R, K), device="cuda") for _ in range(2))
        ids = torch.zeros((s.R, K, 4), dtype=torch.int32, device="cuda")
        lws = torch.zeros(mcd.mcd_logprobs_workspace_bytes(s.R, K, V, 4), dtype=torch.uint8,
                          device="cuda")
        row = i32([a for a, _ in plan.sampled_rows()])
        mcd.mcd_logprobs(scores.view(s.R, K, V), tokens, lp, lws, entropy=H, top_ids=ids,
                         token_row=row, pad_id=s.head.pad_id)
        assert mcd.mcd_read_device_status(lws) == 0
        x, t, order = scores.double().cpu().numpy(), tokens.cpu().numpy(), row.cpu().numpy()
        for i in range(s.R):
            for k in range(K):
                want, ent, top, units, H_units = reference(x[i, k * V:(k + 1) * V], 4)
                tok = t[order[i], k]
                assert (tok == V) == (step < k)      # the delay pattern: no frame yet
                expect, tol = (0.0, 0.0) if tok == V else (want[tok], units[tok] * 2.0 ** -24)
                assert abs(float(lp[i, k]) - expect) <= tol
                assert abs(float(H[i, k]) - ent) <= H_units * 2.0 ** -24
                assert ids[i, k].tolist() == top.tolist()
        s.score.index_add_(0, row.long(), lp.double().sum(1))
        history.append(lp.clone())
        context += 1
    # rank, keep the best of each prompt, give the others' pages back
    best = s.score.view(s.P, s.n).argmax(1).cpu().numpy() + np.arange(s.P) * s.n
    loser = np.setdiff1d(np.arange(s.R), best)
    mcd.mcd_cache_release(s.pages, i32(s.P + loser), s.ws)
    refs, table = s.pages.refs.cpu().numpy(), s.cache.table.cpu().numpy()
    held = table[s.P + best]
    assert refs.sum() == (held >= 0).sum() and (refs[held[held >= 0]] == 1).all()
    mcd.mcd_cache_release(s.pages, i32(s.P + best), s.ws)
    assert not s.pages.refs.any() and bool((s.cache.table == -1).all())
    assert mcd.mcd_read_device_status(s.ws) == 0


def test_captured_steps_take_pages():
    """One captured step (pages, append, attention, log probabilities), replayed while contexts
    advance on the device past pages' ends, against eager steps."""
    results = []
    for graphed in (False, True):
        s = Serving([120, 190], 4, seed=3, steps=8)
        s.prefill()
        s.fork()
        context, one = i32(s.lengths[s.of]), i32(np.ones(s.R))
        start = torch.zeros(s.R + 1, dtype=torch.int32, device="cuda")
        most = s.cache.max_pages * 64
        rows = mcd.CacheRows(context, start=start, slot=s.slot, n_tokens=s.R, max_context=most)
        ws = s.cache.workspace(rows, HQ, groups=s.groups)
        qkv = torch.zeros((s.R, HQ + 2 * HKV, D), dtype=BF16, device="cuda")
        out = torch.zeros((s.R, HQ, D), dtype=BF16, device="cuda")
        lp = torch.zeros((s.R, 1), device="cuda")
        tok = torch.full((s.R, 1), 7, dtype=torch.int32, device="cuda")
        lws = torch.zeros(256, dtype=torch.uint8, device="cuda")

        def step():
            mcd.mcd_cache_reserve(s.pages, context, one, start, s.ws, slot=s.slot, n_tokens=s.R,
                                  max_tokens=1, max_context=most)
            mcd.mcd_cache_append(s.cache, rows, qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], s.ws)
            mcd.mcd_cache_attend_shared(s.cache, rows, s.groups, qkv[:, :HQ], out, ws)
            mcd.mcd_logprobs(out.view(s.R, 1, HQ * D), tok, lp, lws)

        graph, got = None, []
        if graphed:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        for _ in range(s.steps):
            qkv.normal_(generator=s.gen)
            graph.replay() if graphed else step()
            got += [out.clone(), lp.clone()]
            context.add_(1)
            torch.cuda.synchronize()
        got += [s.cache.table.clone(), s.cache.pages.clone(), s.pages.refs.clone()]
        assert [mcd.mcd_read_device_status(w) for w in (ws, s.ws, lws)] == [0, 0, 0]
        results.append(got)
    for a, b in zip(*results):
        assert torch.equal(a, b)
