"""The 4-bit key/value cache on the GPU where its inputs or its use go to the limits: logits and
values of any size, rows that have no token, replays with other rows, workspaces and buffers that
are shared.  Against tests/_cache_ref.py in 64 bits."""
import numpy as np
import pytest

import _cache_ref as ref
import test_gpu_cache as base
from test_gpu_cache import BF16, F32, dev, i32, make_cache, make_rows, rounded, slot_kv, starts

torch = pytest.importorskip("torch")
mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


def fill(cache, k, v):
    """Keys and values [slot][Hkv][L][D] (numpy) into a cache's pages, in order; the host copy of
    the pages and of the table."""
    R, H, L, D = k.shape
    n = -(-L // 64)
    table = np.full(tuple(cache.table.shape), -1, np.int32)
    table[:, :n] = np.arange(R * n)[::-1].reshape(R, n)
    cache.table.copy_(i32(table))
    kt, vt = (dev(x.astype(np.float32)).permute(0, 2, 1, 3).reshape(R * L, H, D).contiguous()
              for x in (k, v))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    mcd.mcd_cache_append(cache, make_rows([0] * R, [L] * R), kt, vt, ws)
    assert mcd.mcd_read_device_status(ws) == 0
    return cache.pages.cpu().numpy(), table


# ---- logits of any size ------------------------------------------------------

LARGE = [
    # name, Hq, Hkv, D, dtype, context, new tokens
    ("kept_scores", 8, 2, 64, BF16, [300, 64, 20, 0], [1, 1, 1, 1]),
    ("kept_scores_fp32", 16, 2, 128, F32, [300, 64, 20, 0], [1, 1, 1, 1]),
    ("single_tile", 32, 2, 64, BF16, [300, 64, 20, 0], [1, 1, 1, 1]),
    ("chunks", 8, 2, 64, BF16, [300, 0, 64], [40, 70, 3]),
    ("chunks_fp32", 4, 2, 64, F32, [300, 0], [40, 70]),
    ("decode_beside_a_prompt", 8, 2, 128, BF16, [300, 0, 64], [1, 70, 1]),
    ("split_row", 4, 1, 64, BF16, [2600], [1]),
    ("split_row_fp32", 4, 1, 64, F32, [2600], [1]),
    ("split_chunk", 4, 1, 64, BF16, [2600], [20]),
]


@pytest.mark.parametrize("name,Hq,Hkv,D,dtype,ctx,new", LARGE, ids=[a[0] for a in LARGE])
def test_large_logits(name, Hq, Hkv, D, dtype, ctx, new):
    """Logits of up to 1.5e31 and of both signs, apart by whole numbers from 0 upwards, so that
    many positions share the weight: outputs, lse and received weight.  Keys of channels 0 and 2
    are 6, of channel 1 a whole number of [-6, 6]; the queries' entries make every score a whole
    number below 2^24 (or a multiple of a power of two, of few bits), which fp32 holds exactly.
    What is left are the exponent (a difference of at most 60 that matters, times log2(e): 3
    roundings), the exponential and the sums: below 128 of 2^-23."""
    rng = np.random.default_rng(sum(map(ord, name)))
    R, N, L = len(ctx), sum(new), max(c + n for c, n in zip(ctx, new))
    k, v = np.zeros((R, Hkv, L, D)), rng.standard_normal((R, Hkv, L, D))
    k[..., 0] = k[..., 2] = 6.0
    k[..., 1] = rng.choice([-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], (R, Hkv, L))
    k[:, :, :L // 2, 1] = np.minimum(k[:, :, :L // 2, 1], -1.0)     # the largest come late
    n_pages = R * -(-L // 64) + 1
    cache = mcd.Cache.alloc(n_pages, Hkv, D, R, -(-L // 64) + 1, weights=True)
    pages, table = fill(cache, k, v)
    # (channel 0, channel 1, channel 2): 2^20 / log2(e) is 726817.2, between the third's logits
    kinds = np.array([(0, 1, 0), (1000, 1, 0), (120832, 1, 304), (121344, 1, 0), (2 ** 17, 1, 0),
                      (2 ** 20, 1, 0), (-2 ** 20, 1, 0), (-120832, -1, -304), (786432, -1, 0),
                      (2490368, 1, 0), (2.0 ** 100, 2.0 ** 100, 0), (-2.0 ** 40, 2.0 ** 40, 0)])
    q = np.zeros((N, Hq, D))
    q[..., :3] = kinds[rng.integers(0, len(kinds), (N, Hq))]
    rows = make_rows(ctx, new)
    qt = dev(q.astype(np.float32)).to(dtype)
    out, wout = torch.full_like(qt, 9.0), torch.full_like(cache.weight, 9.0)
    lse = torch.zeros((N, Hq), device="cuda")
    ws = cache.workspace(rows, Hq)
    print(f"case large logits {name}", flush=True)
    mcd.mcd_cache_attend(cache, rows, qt, out, ws, scale=1.0, lse=lse, weight_out=wout)
    assert mcd.mcd_read_device_status(ws) == 0
    rel = 128 * 2.0 ** -23
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r in range(R):
        a, n = starts(new)[r], new[r]
        kd, vd = slot_kv(pages, table, r, ctx[r] + n, D)
        assert np.array_equal(kd[..., :3], k[r, :, :ctx[r] + n, :3])
        o, l, wt, size = ref.attend(kd, vd, q[a:a + n], ctx[r], 1.0)
        to = (rel + (2.0 ** -8 if dtype == BF16 else 2.0 ** -22)) * size
        w = wout[r, :, :ctx[r] + n].double().cpu().numpy()
        assert (np.abs(w - wt) <= rel * wt + 1e-12).all(), (r, np.abs(w - wt).max())
        assert (np.abs(got[a:a + n] - o) <= to).all(), (r, np.abs(got[a:a + n] - o).max())
        # the reference, log2(e) and the sum: six roundings of 2^-24
        assert (np.abs(got_lse[a:a + n] - l) <= rel + 2.0 ** -21 * np.abs(l)).all()


# ---- start is read when the kernels run --------------------------------------

@pytest.mark.parametrize("Hq", [8, 80], ids=["narrow", "wide"])
def test_replay_with_idle_rows(Hq):
    """A decode step (append, read, attention with weights) captured with a token in every row and
    replayed while some rows are idle: equal starts, fewer tokens than the call's bound."""
    D, H, R = 64, 2, 4
    rng = np.random.default_rng(31)
    ctx0 = [130, 62, 63, 300]
    cache, pages, table, w, _ = make_cache(rng, [c + 3 for c in ctx0], H, D, weights=True)
    context, start = i32(ctx0), i32(np.arange(R + 1))
    rows = mcd.CacheRows(context, start=start, n_tokens=R, max_context=400)
    ws = cache.workspace(rows, Hq)
    qkv = torch.zeros((R, Hq + 2 * H, D), dtype=F32, device="cuda")
    k, v = qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    kr, vr = torch.zeros((R, H, D), device="cuda"), torch.zeros((R, H, D), device="cuda")
    out = torch.zeros((R, Hq, D), device="cuda")

    def step():
        mcd.mcd_cache_append(cache, rows, k, v, ws)
        mcd.mcd_cache_read(cache, rows, kr, vr, ws)
        mcd.mcd_cache_attend(cache, rows, qkv[:, :Hq], out, ws, weight_out=cache.weight)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    length = np.array(ctx0)
    want = w.astype(np.float64)
    for new in ([1, 1, 1, 1], [1, 0, 1, 1], [0, 0, 0, 1], [0, 0, 0, 0]):
        x = rng.standard_normal((R, Hq + 2 * H, D)).astype(np.float32)
        qkv.copy_(dev(x))
        context.copy_(i32(length))
        start.copy_(i32(starts(new)))
        for t in (kr, vr, out):
            t.fill_(9.0)
        print(f"case replay {new}", flush=True)
        graph.replay()
        torch.cuda.synchronize()
        assert mcd.mcd_read_device_status(ws) == 0
        a = starts(new)
        tol_w = np.full(want.shape, 2.0 ** -22) * want
        for r in range(R):
            if new[r]:
                for h in range(H):
                    ref.put(pages[table[r, length[r] // 64], h], D, length[r] % 64,
                            x[a[r], Hq + h], x[a[r], Hq + H + h])
                want[r, :, length[r]] = tol_w[r, :, length[r]] = 0.0
        assert np.array_equal(cache.pages.cpu().numpy(), pages)
        for r in range(R):
            if not new[r]:
                continue
            L = length[r] + 1
            kd, vd = slot_kv(pages, table, r, L, D)
            assert np.array_equal(kr[a[r]].cpu().numpy(), kd[:, -1])
            assert np.array_equal(vr[a[r]].cpu().numpy(), rounded(vd[:, -1], F32))
            q = x[a[r]:a[r] + 1, :Hq].astype(np.float64)
            o, _, wt, size = ref.attend(kd, vd, q, L - 1, 0.125)
            to, tw, _ = base.bounds(kd, q, 0.125, F32, wt, size)
            assert (np.abs(out[a[r]].double().cpu().numpy() - o[0]) <= to).all()
            want[r, :, :L] += wt
            tol_w[r, :, :L] += tw
        got = cache.weight.double().cpu().numpy()
        assert (np.abs(got - want) <= tol_w).all()
        want = got
        assert bool((out[a[-1]:] == 9.0).all()) and bool((kr[a[-1]:] == 9.0).all())
        length = length + new


# ---- rows without a token ----------------------------------------------------

@pytest.mark.parametrize("name,Hq,ctx,new", [
    ("kept_scores", 4, [70, 200, 0, 5], [1, 0, 0, 2]),
    ("single_tile", 32, [70, 200, 0, 5], [1, 0, 0, 1]),
    ("beside_a_prompt", 8, [70, 200, 0, 5], [1, 0, 0, 40]),
    ("wide", 40, [70, 200, 0, 5], [1, 0, 0, 40]),
    ("no_token_at_all", 8, [70, 200, 0, 5], [0, 0, 0, 0]),
])
@pytest.mark.parametrize("cached", [True, False], ids=["weights", "no_weights"])
def test_weight_of_rows_without_a_token(name, Hq, ctx, new, cached):
    """weight_out holds what they had received before, or 0 of a cache without weights; in place
    they keep it."""
    rng = np.random.default_rng(len(name))
    D, H, R, N = 64, 2, 4, sum(new)
    slot = [2, 0, 3, 1]
    lengths = np.zeros(R, int)
    lengths[slot] = np.array(ctx) + new
    cache, pages, table, w, _ = make_cache(rng, lengths, H, D, weights=cached)
    rows = make_rows(ctx, new, slot)
    q = dev(rng.standard_normal((max(N, 1), Hq, D)).astype(np.float32)).to(BF16)
    shape = (R, H, table.shape[1] * 64)
    wout = torch.full(shape, 9.0, device="cuda")
    ws = cache.workspace(rows, Hq)
    print(f"case no token {name} {cached}", flush=True)
    mcd.mcd_cache_attend(cache, rows, q, torch.zeros_like(q), ws, weight_out=wout)
    assert mcd.mcd_read_device_status(ws) == 0
    for r in range(R):
        if new[r] == 0:
            got = wout[slot[r]].cpu().numpy()
            want = w[slot[r]] if cached else np.zeros(shape[1:])
            assert np.array_equal(got[:, :ctx[r]], want[:, :ctx[r]])
            assert (got[:, ctx[r]:] == 9.0).all()
    if cached:
        mcd.mcd_cache_attend(cache, rows, q, torch.zeros_like(q), ws, weight_out=cache.weight)
        got = cache.weight.cpu().numpy()
        for r in range(R):
            if new[r] == 0:
                assert np.array_equal(got[slot[r]], w[slot[r]])


# ---- one workspace -----------------------------------------------------------

def test_one_workspace_for_every_smaller_step():
    """A workspace sized once, for the largest step: fewer and longer rows (split and joined), kept
    scores, chunks.  The same bits as with a workspace of their own, and nothing written past the
    size that the largest step asked for."""
    rng = np.random.default_rng(17)
    H, D, Hq = 2, 64, 8
    cache, *_ = make_cache(rng, [3000] * 4 + [200] * 60, H, D, weights=True)
    most = mcd.CacheRows(i32([0] * 64), start=i32(np.arange(65)), n_tokens=300, max_tokens=40,
                         max_context=3000)
    size = mcd.mcd_cache_workspace_bytes(cache, most, Hq)
    buf = torch.full((size + 4096,), 171, dtype=torch.uint8, device="cuda")
    buf[:256] = 0
    for ctx, new in (([2999], [1]), ([2900, 100], [40, 1]), ([150] * 60, [1] * 60), ([2000], [3]),
                     ([2500, 0, 1000], [2, 2, 2]), ([100, 50, 0], [0, 7, 1])):
        rows, N = make_rows(ctx, new), sum(new)
        q = dev(rng.standard_normal((N, Hq, D)).astype(np.float32)).to(BF16)
        got = []
        print(f"case one workspace {ctx[:3]} {new[:3]}", flush=True)
        for ws in (buf[:size], cache.workspace(rows, Hq)):
            out, wout = torch.zeros_like(q), torch.zeros_like(cache.weight)
            mcd.mcd_cache_attend(cache, rows, q, out, ws, weight_out=wout)
            assert mcd.mcd_read_device_status(ws) == 0
            got.append((out, wout))
        assert all(torch.equal(a, b) for a, b in zip(*got))
        assert bool((buf[size:] == 171).all())


# ---- values that are not finite, and the largest -----------------------------

@pytest.mark.parametrize("n", [1, 40], ids=["decode", "chunk"])
@pytest.mark.parametrize("Hq", [4, 8, 16, 32])
def test_value_that_is_not_finite_at_a_weight_of_nearly_nothing(Hq, n):
    """A softmax weight below what fp32 holds is still a weight: what sees the position is NaN, in
    a full page as in the last one, and what does not see it is not."""
    D, H, ctx = 64, 2, 200
    for at in (30, 195, ctx + n // 2):
        k, v = np.full((1, H, ctx + n, D), -6.0), np.ones((1, H, ctx + n, D))
        k[:, :, 3] = 6.0                                      # the only one that has any weight
        v[0, 1, at, 5] = np.nan
        cache = mcd.Cache.alloc(6, H, D, 1, 5, weights=True)
        fill(cache, k, v)
        q = torch.full((n, Hq, D), 2.0, dtype=BF16, device="cuda")
        rows = make_rows([ctx], [n])
        out, lse = torch.zeros_like(q), torch.zeros((n, Hq), device="cuda")
        wout = torch.zeros_like(cache.weight)
        ws = cache.workspace(rows, Hq)
        print(f"case nearly no weight Hq={Hq} n={n} at={at}", flush=True)
        mcd.mcd_cache_attend(cache, rows, q, out, ws, scale=1.0, lse=lse, weight_out=wout)
        nan = torch.isnan(out).cpu().numpy()
        sees = ctx + np.arange(n) >= at
        assert not nan[:, :Hq // 2].any()
        assert nan[sees][:, Hq // 2:].all() and not nan[~sees].any()
        assert bool(torch.isfinite(lse).all())
        w = wout[0, :, :ctx + n].cpu().numpy()
        want = np.where(np.arange(ctx + n) == 3, n * Hq // H, 0.0)
        assert (np.abs(w - want) <= 2.0 ** -20 * want).all()


HUGE = [
    # name, Hq, Hkv, D, dtype, context, new tokens
    ("decode", 8, 2, 64, BF16, [700, 64, 20, 0], [1, 1, 1, 1]),
    ("decode_fp32", 4, 2, 128, F32, [700, 64, 20, 0], [1, 1, 1, 1]),
    ("groups_of_eight", 16, 2, 64, BF16, [700, 64, 20, 0], [1, 1, 1, 1]),
    ("groups_of_sixteen", 32, 2, 64, BF16, [700, 64, 20, 0], [1, 1, 1, 1]),
    ("groups_of_sixteen_fp32", 32, 2, 64, F32, [700, 64, 20, 0], [1, 1, 1, 1]),
    ("wide_heads", 4, 2, 256, BF16, [100, 3], [1, 30]),
    ("chunks", 8, 2, 128, BF16, [300, 0], [40, 70]),
    ("chunks_fp32", 4, 2, 64, F32, [300, 0], [40, 70]),
    ("split_row", 4, 1, 64, BF16, [2600], [1]),
    ("split_chunk_fp32", 4, 1, 64, F32, [2600], [20]),
]


@pytest.mark.parametrize("where", ["all", "some", "late"])
@pytest.mark.parametrize("name,Hq,Hkv,D,dtype,ctx,new", HUGE, ids=[a[0] for a in HUGE])
def test_largest_values(name, Hq, Hkv, D, dtype, ctx, new, where):
    """Values of up to 6 * 2^125 = 2.6e38, whose weighted sum fits the type though their sum does
    not: everywhere, at a few positions, and after ordinary ones.  The bounds are those of every
    other value."""
    rng = np.random.default_rng(sum(map(ord, name + where)))
    R, N, L = len(ctx), sum(new), max(c + n for c, n in zip(ctx, new))
    k = rng.standard_normal((R, Hkv, L, D))
    v = rng.choice([-6.0, -3, 0, 1, 4, 6], (R, Hkv, L, D), p=[.1, .1, .1, .1, .2, .4])
    v[..., 0] = 6.0
    large = {"all": np.ones(L, bool), "some": np.arange(L) % 37 == 5,
             "late": np.arange(L) >= 0.8 * L}[where]
    v *= np.where(large, 2.0 ** 125, 1.0)[:, None]
    cache = mcd.Cache.alloc(R * -(-L // 64) + 1, Hkv, D, R, -(-L // 64) + 1, weights=True)
    pages, table = fill(cache, k, v)
    q = rounded(rng.standard_normal((N, Hq, D)) * 2, dtype)
    rows = make_rows(ctx, new)
    qt = dev(q).to(dtype)
    out, wout = torch.zeros_like(qt), torch.zeros_like(cache.weight)
    lse = torch.zeros((N, Hq), device="cuda")
    ws = cache.workspace(rows, Hq)
    print(f"case largest values {name} {where}", flush=True)
    mcd.mcd_cache_attend(cache, rows, qt, out, ws, scale=0.125, lse=lse, weight_out=wout)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r in range(R):
        a, n = starts(new)[r], new[r]
        kd, vd = slot_kv(pages, table, r, ctx[r] + n, D)
        o, l, wt, size = ref.attend(kd, vd, q[a:a + n].astype(np.float64), ctx[r], 0.125)
        to, tw, tl = base.bounds(kd, q[a:a + n], 0.125, dtype, wt, size)
        assert (np.abs(got[a:a + n] - o) <= to).all(), r
        w = wout[r, :, :ctx[r] + n].double().cpu().numpy()
        assert (np.abs(w - wt) <= tw).all()
        # the logarithm and the reference, both up to 70, cancel: 4 roundings of 2^-18
        assert (np.abs(got_lse[a:a + n] - l) <= tl + 2.0 ** -22 * np.abs(l) + 2.0 ** -16).all()


# ---- the caller's buffers ----------------------------------------------------

@pytest.mark.parametrize("Hq", [8, 16, 32])
def test_weights_that_begin_at_any_float(Hq):
    """weight and weight_out may be views into larger buffers, at any float."""
    rng = np.random.default_rng(5)
    H, D, ctx, new = 2, 64, [300, 64, 5], [1, 1, 1]
    cache, pages, table, w, _ = make_cache(rng, [c + 1 for c in ctx], H, D, weights=True)
    rows = make_rows(ctx, new)
    q = dev(rng.standard_normal((3, Hq, D)).astype(np.float32)).to(BF16)
    want = None
    for shift in (0, 1, 2, 3):
        buf = torch.zeros((2, w.size + 4), device="cuda")
        win, wout = (b[shift:shift + w.size].view(w.shape) for b in buf)
        win.copy_(dev(w))
        here = mcd.Cache(cache.pages, cache.table, D, win)
        ws = here.workspace(rows, Hq)
        out = torch.zeros_like(q)
        print(f"case weights at float {shift} Hq={Hq}", flush=True)
        mcd.mcd_cache_attend(here, rows, q, out, ws, weight_out=wout)
        assert mcd.mcd_read_device_status(ws) == 0
        want = wout.clone() if want is None else want
        assert torch.equal(wout, want) and torch.equal(win, dev(w))
        assert bool((buf[:, :shift] == 0).all()) and bool((buf[:, shift + w.size:] == 0).all())


def test_out_beside_and_in_place_of_the_queries():
    """q and out may be columns of one buffer; without weight_out they may be the same."""
    rng = np.random.default_rng(6)
    H, D, Hq, ctx, new = 2, 64, 8, [300, 0, 5], [1, 40, 1]
    cache, *_ = make_cache(rng, [c + n for c, n in zip(ctx, new)], H, D, weights=True)
    rows, N = make_rows(ctx, new), sum(new)
    buf = torch.zeros((N, 2 * Hq, D), dtype=BF16, device="cuda")
    q = dev(rng.standard_normal((N, Hq, D)).astype(np.float32)).to(BF16)
    buf[:, :Hq] = q
    ws = cache.workspace(rows, Hq)
    out, wout = torch.zeros_like(q), torch.zeros_like(cache.weight)
    wout2 = torch.zeros_like(wout)
    mcd.mcd_cache_attend(cache, rows, q, out, ws, weight_out=wout)
    mcd.mcd_cache_attend(cache, rows, buf[:, :Hq], buf[:, Hq:], ws, weight_out=wout2)
    assert torch.equal(buf[:, Hq:], out) and torch.equal(wout, wout2)
    assert torch.equal(buf[:, :Hq], q)
    mcd.mcd_cache_attend(cache, rows, buf[:, :Hq], buf[:, :Hq], ws)
    assert torch.equal(buf[:, :Hq], out)
    with pytest.raises(mcd.McdError) as e:
        mcd.mcd_cache_attend(cache, rows, q, q, ws, weight_out=wout)
    assert e.value.code == mcd.MCD_E_INVALID


# ---- every tile of few query rows --------------------------------------------

@pytest.mark.parametrize("weights", [False, True], ids=["plain", "weights"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("name,Hq,Hkv,ctx,new", [
    ("three_heads", 3, 1, [2500, 63, 0, 700], [1, 1, 1, 1]),
    ("five_heads", 10, 2, [2500, 63, 0, 700], [1, 1, 1, 1]),
    ("eight_heads", 8, 1, [2500, 63, 0, 700], [1, 1, 1, 1]),
    ("eight_heads_two_tokens", 8, 1, [1300, 62, 0], [2, 2, 1]),
    ("eleven_heads", 22, 2, [1300, 63, 0], [1, 1, 1]),
    ("sixteen_heads", 16, 1, [2500, 63, 0, 700], [1, 1, 1, 1]),
    ("sixteen_heads_beside_a_prompt", 16, 1, [200, 0, 63], [1, 20, 1]),
])
def test_narrow_tiles(name, Hq, Hkv, ctx, new, D, dtype, weights):
    base.test_attend(name, Hq, Hkv, D, dtype, ctx, new, weights)


def test_no_row_sees_a_position():
    """Rows that see nothing at all: bounds of no position, with every output."""
    H, D, Hq = 2, 64, 8
    cache = mcd.Cache.alloc(3, H, D, 2, 2, weights=True)
    cache.weight.fill_(3.0)
    for ctx, new in (([-1, -1], [1, 1]), ([-3, -40], [3, 40])):
        rows, N = make_rows(ctx, new), sum(new)
        q = torch.ones((N, Hq, D), dtype=BF16, device="cuda")
        out, lse = torch.full_like(q, 9.0), torch.zeros((N, Hq), device="cuda")
        wout = torch.full_like(cache.weight, 5.0)
        ws = cache.workspace(rows, Hq)
        mcd.mcd_cache_attend(cache, rows, q, out, ws, lse=lse, weight_out=wout)
        assert mcd.mcd_read_device_status(ws) == 0
        assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())
        assert bool((wout == 5.0).all())


# ---- the types' whole range --------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 90], ids=["one", "chunk"])
def test_append_over_the_types_range(n, dtype):
    """Keys and values from the smallest subnormal numbers to the largest, bytes and values."""
    rng = np.random.default_rng(n)
    D, H, R = 64, 2, 60 if n == 1 else 2
    ctx, new = [int(c) for c in rng.integers(0, 70, R)], [n] * R
    cache, pages, table, _, _ = make_cache(rng, [c + n for c in ctx], H, D)
    N = R * n
    with np.errstate(over="ignore"):
        x = (rng.uniform(1, 2, (N, 2 * H, D)) * rng.choice([-1, 1], (N, 2 * H, D))
             * np.exp2(rng.integers(-3, 1, (N, 2 * H, D)))).astype(np.float64) \
            * np.exp2(rng.integers(-149, 128, (N, 2 * H, 1)).astype(np.float64))
        x = rounded(np.clip(x, -3.38e38, 3.38e38), dtype)
    x[0] = np.float32(1e-45) if dtype == F32 else rounded(9.2e-41, dtype)
    t = dev(x).to(dtype)
    assert torch.equal(t.float().cpu(), torch.from_numpy(x))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    rows = make_rows(ctx, new)
    print(f"case append range n={n} {dtype}", flush=True)
    mcd.mcd_cache_append(cache, rows, t[:, :H], t[:, H:], ws)
    kr, vr = (torch.full((N, H, D), 7.0, device="cuda") for _ in range(2))
    mcd.mcd_cache_read(cache, rows, kr, vr, ws)
    got_k, got_v = kr.cpu().numpy(), vr.cpu().numpy()
    for r in range(R):
        for i in range(n):
            pos, tok = ctx[r] + i, starts(new)[r] + i
            for h in range(H):
                page = pages[table[r, pos // 64], h]
                ref.put(page, D, pos % 64, x[tok, h], x[tok, H + h])
                k, v = ref.get(page, D, pos % 64)
                assert np.array_equal(got_k[tok, h], k.astype(np.float32)), (tok, h)
                assert np.array_equal(got_v[tok, h], v.astype(np.float32)), (tok, h)
    assert np.array_equal(cache.pages.cpu().numpy(), pages)


@pytest.mark.parametrize("ks,vs", [(-90, -90), (100, 60), (-60, 63), (90, 64), (-100, 124)])
@pytest.mark.parametrize("name,Hq,dtype,ctx,new", [
    ("decode", 8, BF16, [700, 20], [1, 1]), ("decode_fp32", 8, F32, [700, 20], [1, 1]),
    ("chunk", 4, BF16, [300, 0], [30, 9]), ("chunk_fp32", 4, F32, [300, 0], [30, 9]),
])
def test_small_and_large_keys_and_values(name, Hq, dtype, ctx, new, ks, vs):
    """Keys times 2^ks with queries times 2^-ks, values times 2^vs: powers of two change nothing,
    so the bounds are those of ordinary numbers, times 2^vs."""
    rng = np.random.default_rng(sum(map(ord, name)))
    R, N, L, H, D = len(ctx), sum(new), max(c + n for c, n in zip(ctx, new)), 2, 64
    k, v = (rng.standard_normal((R, H, L, D)) for _ in range(2))
    cache = mcd.Cache.alloc(R * -(-L // 64) + 1, H, D, R, -(-L // 64) + 1, weights=True)
    pages, table = fill(cache, k * 2.0 ** ks, v * 2.0 ** vs)
    q = rounded(rng.standard_normal((N, Hq, D)) * 2.0, dtype)
    rows = make_rows(ctx, new)
    qt = dev(q * np.float32(2.0 ** -ks)).to(dtype)
    out, wout = torch.zeros_like(qt), torch.zeros_like(cache.weight)
    ws = cache.workspace(rows, Hq)
    print(f"case small and large {name} {ks} {vs}", flush=True)
    mcd.mcd_cache_attend(cache, rows, qt, out, ws, scale=0.125, weight_out=wout)
    assert mcd.mcd_read_device_status(ws) == 0
    got = out.double().cpu().numpy()
    for r in range(R):
        a, n = starts(new)[r], new[r]
        kd, vd = slot_kv(pages, table, r, ctx[r] + n, D)
        kd, vd = kd * 2.0 ** -ks, vd * 2.0 ** -vs
        o, _, wt, size = ref.attend(kd, vd, q[a:a + n].astype(np.float64), ctx[r], 0.125)
        to, tw, _ = base.bounds(kd, q[a:a + n], 0.125, dtype, wt, size)
        assert (np.abs(got[a:a + n] * 2.0 ** -vs - o) <= to).all(), r
        w = wout[r, :, :ctx[r] + n].double().cpu().numpy()
        assert (np.abs(w - wt) <= tw).all()


def test_starts_that_do_not_begin_at_zero():
    """Tokens before the first row's belong to no row: no call reads or writes for them, and the
    rows' own have their results."""
    rng = np.random.default_rng(31)
    D, H, Hq, ctx, new, first = 64, 2, 4, [70, 3, 130], [2, 1, 40], 45
    lengths = [c + n for c, n in zip(ctx, new)]
    cache, pages, table, _, _ = make_cache(rng, lengths, H, D)
    N = sum(new)
    start = first + np.concatenate([[0], np.cumsum(new)])
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    q = dev(rng.standard_normal((first + N, Hq, D)).astype(np.float32))
    kv = dev(rng.standard_normal((first + N, 2 * H, D)).astype(np.float32))

    def rows(begin):
        return mcd.CacheRows(i32(ctx), start=i32(start - first + begin), n_tokens=begin + N,
                             max_tokens=max(new), max_context=max(lengths))

    outs = []
    for begin in (0, first):
        cache.pages.copy_(dev(pages))
        out, ko, vo = (torch.full((begin + N, h, D), 9.0, device="cuda") for h in (Hq, H, H))
        part = slice(first - begin, None)
        mcd.mcd_cache_append(cache, rows(begin), kv[part, :H], kv[part, H:], ws)
        mcd.mcd_cache_read(cache, rows(begin), ko, vo, ws)
        mcd.mcd_cache_attend(cache, rows(begin), q[part], out, ws)
        assert mcd.mcd_read_device_status(ws) == 0
        for x in (out, ko, vo):
            assert bool((x[:begin] == 9.0).all())
        outs.append([x[begin:].clone() for x in (out, ko, vo)] + [cache.pages.clone()])
    for a, b in zip(*outs):
        # other splits of the pages: exponents of up to 64 are rounded against another reference,
        # 2^-18 twice, and the sums are added in another order, 16 of 2^-23, of values up to 6
        assert torch.allclose(a.float(), b.float(), rtol=0, atol=6 * 2.0 ** -16, equal_nan=True)
