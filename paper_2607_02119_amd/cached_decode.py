"""The 4-bit key/value cache in the decode loop: scheduler, cache, head.

    python -m paper_2607_02119_amd.cached_decode --steps 200 --rows 64 --bound 256

Requests in flight (half of them guided pairs) go through the paired scheduler.
Every planned step runs one attention layer over the cache for all its rows,
prompt chunks and decoding rows alike: the inputs' queries, keys and values
(``mcd_next_input`` for rows that decode, random embeddings for prompts, a random
projection), ``mcd_cache_append``, ``mcd_cache_attend`` with the received weight.
The decoding rows' outputs are the hidden states of the head step, whose tokens
make the next inputs.  A Companion that joins after its request's text phase
starts with a copy of its Main row's cache, and a row whose cache outgrows
``bound`` positions keeps ``keep`` of them (both ``mcd_cache_evict``).

The model is a stand-in of random weights; the bookkeeping around the calls (page
lists, the table, lengths) is what a serving program does.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import mcd

PAGE = mcd.MCD_CACHE_PAGE


class PagePool:
    """Free pages, the pages and length of every slot, and the table's host copy."""

    def __init__(self, n_pages, n_slots, max_pages):
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages = [[] for _ in range(n_slots)]
        self.length = np.zeros(n_slots, np.int64)
        self.table = np.full((n_slots, max_pages), -1, np.int32)

    def take(self, n):
        if n > len(self.free):
            raise RuntimeError("the cache has no page left")
        return [self.free.pop() for _ in range(n)]

    def set(self, slot, pages, length):
        self.free.extend(p for p in self.pages[slot] if p not in pages)
        self.pages[slot], self.length[slot] = list(pages), length
        self.table[slot] = -1
        self.table[slot, :len(pages)] = pages

    def grow(self, slot, length):
        need = -(-int(length) // PAGE) - len(self.pages[slot])
        self.set(slot, self.pages[slot] + self.take(max(need, 0)), length)


class CachedDecode:
    def __init__(self, rows=64, bound=256, keep=192, recent=64, Hq=8, Hkv=2, D=128, K=4, V=256,
                 V_text=512, null_prompt=4, seed=0, device="cuda"):
        self.rows, self.bound, self.keep, self.recent = rows, bound, keep, recent
        self.Hq, self.Hkv, self.D, self.K, self.V, self.V_text = Hq, Hkv, D, K, V, V_text
        self.device, self.rng = device, np.random.default_rng(seed)
        gen = torch.Generator(device=device).manual_seed(seed)
        H = self.H = Hq * D

        def normal(*shape, scale=1.0):
            return (torch.randn(shape, generator=gen, device=device) * scale).to(torch.bfloat16)

        self.W_qkv = normal(H, (Hq + 2 * Hkv) * D, scale=H ** -0.5)
        self.budget = 8 * rows                 # tokens of a step at most
        self.E, self.E_text = normal(K, V + 1, H, scale=K ** -0.5), normal(V_text, H)
        self.prompt = normal(max(self.budget, 4096), H)
        self.head = mcd.Head(normal(K, V, H, scale=H ** -0.5), np.arange(K), V,
                             W_text=normal(V_text, H, scale=H ** -0.5))
        self.sched = mcd.Scheduler(rows, self.budget, null_prompt, K - 1, max_requests=2 * rows)
        # every slot up to its bound and a prompt chunk more, twice over for what moves
        longest = bound + self.budget
        max_pages = -(-longest // PAGE) + 1
        n_pages = rows * (-(-bound // PAGE) + 2) + 2 * max_pages + rows * (-(-keep // PAGE))
        self.pool = PagePool(n_pages, rows, max_pages)
        self.cache = mcd.Cache.alloc(n_pages, Hkv, D, rows, max_pages, weights=True, device=device)
        self.next_in = torch.zeros((rows, H), dtype=torch.bfloat16, device=device)   # by slot
        self.null_prompt = null_prompt
        self.workspace = torch.zeros(256, dtype=torch.uint8, device=device)
        self.reported = 0                      # status bits of workspaces that were replaced
        self.head_workspace = self.head.workspace(rows, device)
        self.frames = 64
        self.grid = torch.full((rows, K, self.frames), -1, dtype=torch.int32, device=device)
        self.evicted = self.copied = 0
        for i in range(rows):
            self.submit()

    def submit(self):
        r = self.rng
        self.sched.submit(3.0 if r.random() < 0.5 else 1.0, int(r.integers(5, 300)),
                          int(r.integers(0, 40)), int(r.integers(20, self.frames)))

    def _i32(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(self.device)

    def move(self, src_slots, dst_slots, keep, recent):
        """The kept positions of src slots into pages of their own, as the dst slots'."""
        pool, n = self.pool, len(src_slots)
        length = pool.length[src_slots]
        new_len = np.minimum(length, keep)
        pages = [pool.take(-(-int(m) // PAGE)) for m in new_len]
        table = np.full((n, max(max(map(len, pages)), 1)), -1, np.int32)
        for r, p in enumerate(pages):
            table[r, :len(p)] = p
        to = mcd.Cache(self.cache.pages, self._i32(table), self.D,
                       torch.zeros((n, self.Hkv, table.shape[1] * PAGE), device=self.device))
        self.cache.table.copy_(self._i32(pool.table))
        kept = torch.empty((n, self.Hkv, keep), dtype=torch.int32, device=self.device)
        mcd.mcd_cache_evict(self.cache, to, self._i32(length), keep, recent, kept,
                            torch.empty(n, dtype=torch.int32, device=self.device),
                            self.workspace, int(length.max()), slot=self._i32(src_slots))
        for r, slot in enumerate(dst_slots):
            pool.set(slot, pages[r], int(new_len[r]))
            self.cache.weight[slot, :, :to.weight.shape[2]] = to.weight[r]
        return kept

    def step(self, check=None):
        """One planned step; check(self, rows, q, out) sees the attention's inputs and outputs.
        Returns the number of decoding rows."""
        b, pool = self.sched.plan(), self.pool
        slot, new = b["row_slot"], b["row_tokens"]
        if not len(slot):
            self.sched.commit()
            return 0
        for i in np.flatnonzero(b["row_context"] == 0):
            pool.set(slot[i], [], 0)
        # Companions at their first audio step whose context has grown meanwhile
        # (their Main row's text): a copy of the Main row's cache
        first = (b["row_kind"] == mcd.MCD_ROW_UNCOND) & (b["step"] == 0)
        join = b["head_row"][first]
        join = join[b["row_context"][join] > self.null_prompt]
        if len(join):
            main = {q: t for q, t, m in zip(b["row_req"], slot, b["row_member"]) if m == 0}
            mains = np.array([main[q] for q in b["row_req"][join]])
            self.move(mains, slot[join], int(max(pool.length[mains].max(), 1)), 0)
            self.copied += len(join)
        context = pool.length[slot].copy()
        for i in range(len(slot)):
            pool.grow(slot[i], context[i] + new[i])
        self.cache.table.copy_(self._i32(pool.table))
        start = np.concatenate([[0], np.cumsum(new)])
        N = int(start[-1])
        x = self.prompt[:N].clone()
        decoding = np.flatnonzero(np.isin(np.arange(len(slot)), b["head_row"]))
        if len(decoding):
            x[self._i32(start[decoding]).long()] = self.next_in[self._i32(slot[decoding]).long()]
        qkv = (x @ self.W_qkv).view(N, self.Hq + 2 * self.Hkv, self.D)
        q, k = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv]
        v = qkv[:, self.Hq + self.Hkv:]
        out = torch.empty((N, self.Hq, self.D), dtype=torch.bfloat16, device=self.device)
        rows = mcd.CacheRows(self._i32(context), start=self._i32(start), slot=self._i32(slot),
                             n_tokens=N, max_tokens=int(new.max()),
                             max_context=int((context + new).max()))
        need = mcd.mcd_cache_workspace_bytes(self.cache, rows, self.Hq)
        if need > self.workspace.numel():
            self.reported |= mcd.mcd_read_device_status(self.workspace)
            self.workspace = torch.zeros(2 * need, dtype=torch.uint8, device=self.device)
        mcd.mcd_cache_append(self.cache, rows, k, v, self.workspace)
        mcd.mcd_cache_attend(self.cache, rows, q, out, self.workspace,
                             weight_out=self.cache.weight)
        if check:
            check(self, b, context, q, out)
        over = slot[(context + new) > self.bound]
        if len(over):
            self.move(over, over, self.keep, self.recent)
            self.evicted += len(over)
        R = b["R"]
        if R:
            self._head(b, out[self._i32(start[b["head_row"]]).long()].reshape(R, self.H))
        for _ in self.sched.commit():
            self.submit()
        return R

    def _head(self, b, hidden):
        R, dev = b["R"], self.device
        plan = self.head.plan(b["pair_map"], b["row_kind"], dev)
        full = lambda v, dt: torch.full((R,), v, dtype=dt, device=dev)  # noqa: E731
        tokens = torch.empty((R, self.K), dtype=torch.int32, device=dev)
        mcd.mcd_head_step(
            self.head.handle, R=R, counts=plan.counts, plan=plan.dev, hidden=hidden.contiguous(),
            cfg_w=torch.from_numpy(b["cfg_w"]).to(dev), temperature=full(1.0, torch.float32),
            top_k=full(50, torch.int32), top_p=full(1.0, torch.float32),
            rng_key=torch.from_numpy(b["row_req"][b["head_row"]].astype(np.int64)).to(dev),
            step=self._i32(b["step"]), n_frames=self._i32(b["n_frames"]),
            grid_slot=self._i32(b["grid_slot"]), seed=7, tokens_out=tokens, frame_grid=self.grid,
            n_slots=self.rows, F_max=self.frames,
            scores=torch.empty((max(plan.Rs, 1), self.K * self.V), device=dev),
            workspace=self.head_workspace)
        nxt = torch.empty((R, self.H), dtype=torch.bfloat16, device=dev)
        mcd.mcd_next_input(self.E, tokens, torch.from_numpy(b["row_kind"]).to(dev), self.V, nxt,
                           E_text=self.E_text, workspace=self.head_workspace)
        self.next_in[self._i32(b["row_slot"][b["head_row"]]).long()] = nxt
        self.tokens = tokens

    def status(self):
        """Device status bits of all steps since the last call."""
        bits, self.reported = self.reported, 0
        return bits | mcd.mcd_read_device_status(self.workspace) | \
            mcd.mcd_read_device_status(self.head_workspace)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--rows", type=int, default=64)
    ap.add_argument("--bound", type=int, default=256)
    args = ap.parse_args()
    loop = CachedDecode(rows=args.rows, bound=args.bound, keep=args.bound * 3 // 4,
                        recent=args.bound // 4)
    t0, decoded = time.perf_counter(), 0
    for i in range(args.steps):
        decoded += loop.step()
        if i % 50 == 49:
            torch.cuda.synchronize()
            print(f"step {i + 1}: {decoded} rows decoded, {loop.copied} Companions copied, "
                  f"{loop.evicted} evictions, {len(loop.pool.free)} pages free", flush=True)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t0) / max(args.steps, 1) * 1e3
    print(f"{ms:.2f} ms a step, device status {loop.status()}")


if __name__ == "__main__":
    main()
