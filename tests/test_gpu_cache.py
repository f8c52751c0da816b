"""The 4-bit key/value cache on the GPU against its plain description in 64 bits
(tests/_cache_ref.py): page bytes and positions kept exactly, attention and received weights
within bounds derived from the roundings."""
import math

import numpy as np
import pytest

import _cache_ref as ref

torch = pytest.importorskip("torch")
mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

BF16, F32 = torch.bfloat16, torch.float32


def dev(a, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype).to("cuda")


def i32(a):
    return dev(np.asarray(a, np.int32))


def rounded(x, dtype):
    """numpy float32 values that dtype holds."""
    return torch.from_numpy(np.asarray(x, np.float32)).to(dtype).float().numpy()


def make_cache(rng, lengths, Hkv, D, weights=False, spare=0, fill=None, max_pages=None):
    """A cache whose slots hold random codes and scales at every position, garbage (scales that
    are not finite included) past a slot's length, pages in no order; and its host copy."""
    counts = [-(-n // 64) for n in lengths]
    cols = max_pages or max(max(counts), 1) + 1
    n_pages = sum(counts) + spare + 2
    pages = rng.integers(0, 256, (n_pages, Hkv, ref.page_bytes(D)), dtype=np.uint8)
    t, nb = np.arange(64), D // 32
    # scales: keys around 2^-1, values around 2^-2 as bfloat16 of any mantissa
    pages[..., 64 * D:66 * D] = rng.integers(124, 128, (n_pages, Hkv, 2 * D))
    vs = rng.uniform(0.1, 0.6, (n_pages, Hkv, 64)).astype(np.float32)
    bits = (ref.bf16_round(vs).view(np.uint32) >> 16).astype(np.uint16)
    pages[..., 66 * D:] = bits.view(np.uint8).reshape(n_pages, Hkv, 128)
    table = np.full((len(lengths), cols), -1, np.int32)
    ids, at = rng.permutation(n_pages), 0
    key = 64 * D + (t % 16)[:, None] * nb * 4 + np.arange(nb)[None] * 4 + (t // 16)[:, None]
    val = 66 * D + 2 * (t // 4 % 4 * 16 + t // 16 * 4 + t % 4)
    for s, (n, c) in enumerate(zip(lengths, counts)):
        table[s, :c] = ids[at:at + c]
        at += c
        if n % 64:
            p = table[s, n // 64]
            for h in range(Hkv):
                pages[p, h, key[n % 64:].ravel()] = 255
                pages[p, h, val[n % 64:]] = 0xC0 if h % 2 else 0x80
                pages[p, h, val[n % 64:] + 1] = 0x7F
    w = rng.exponential(1.0, (len(lengths), Hkv, cols * 64)).astype(np.float32) if weights else None
    cache = mcd.Cache(dev(pages), i32(table), D, None if w is None else dev(w))
    return cache, pages, table, w, ids[at:]


def slot_kv(pages, table, s, n, D):
    """Keys, values [Hkv, n, D] of a slot in float64."""
    H = pages.shape[1]
    if n == 0:
        return np.zeros((H, 0, D)), np.zeros((H, 0, D))
    k, v = ref.decode_pages(pages[table[s, :-(-n // 64)]], D)
    return [x.transpose(1, 0, 2, 3).reshape(H, -1, D)[:, :n] for x in (k, v)]


def starts(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def make_rows(ctx, new, slot=None, start=True, max_context=None, max_tokens=None):
    total = [c + n for c, n in zip(ctx, new)]
    return mcd.CacheRows(i32(ctx), start=i32(starts(new)) if start else None,
                         slot=None if slot is None else i32(slot), n_tokens=int(sum(new)),
                         max_tokens=max(new) if max_tokens is None else max_tokens,
                         max_context=max(max(total), 0) if max_context is None else max_context)


# ---- append and read ---------------------------------------------------------

APPENDS = [
    # name, Hkv, D, dtype, steps of (context, new tokens) of every row
    ("one_token", 1, 64, BF16, [([0], [1])]),
    ("decode_steps", 2, 128, BF16, [([61, 0, 127], [1, 1, 1]), ([62, 1, 128], [1, 1, 1]),
                                    ([63, 2, 129], [1, 1, 1]), ([64, 3, 130], [1, 1, 1])]),
    ("rows_without_a_token", 3, 64, F32, [([5, 70, 0, 9], [1, 0, 1, 0])]),
    ("odd_chunks", 2, 128, BF16, [([3, 64, 31, 0], [30, 7, 66, 1]), ([33, 71, 97, 1], [1, 0, 2, 95])]),
    ("across_pages_fp32", 1, 128, F32, [([63, 0], [2, 129])]),
    ("wide_heads", 2, 256, BF16, [([17, 40], [48, 1]), ([65, 41], [1, 1])]),
    ("wide_heads_fp32", 1, 256, F32, [([0], [33])]),
    ("many_heads", 9, 64, BF16, [([10, 0, 3], [5, 11, 2])]),
]


@pytest.mark.parametrize("name,Hkv,D,dtype,steps", APPENDS, ids=[a[0] for a in APPENDS])
def test_append_bytes_and_read(name, Hkv, D, dtype, steps):
    rng = np.random.default_rng(len(name) * 7 + D)
    R = len(steps[0][0])
    lengths = [max(c[r] + n[r] for c, n in steps) for r in range(R)]
    cache, pages, table, w, _ = make_cache(rng, lengths, Hkv, D, weights=True)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    for step, (ctx, new) in enumerate(steps):
        N = sum(new)
        # tokens beside each other's queries, as a fused projection leaves them
        x = rng.standard_normal((max(N, 1), 3 * Hkv, D)).astype(np.float32) \
            * np.exp2(rng.integers(-12, 12, (max(N, 1), 3 * Hkv, 1)))
        x = rounded(x, dtype)
        x[0, Hkv] = x[0, 3 * Hkv - 1] = 0.0                       # heads of zeros
        if N > 1:
            x[1, Hkv] = np.resize(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]), D)
            x[1, 2 * Hkv] = -x[1, Hkv]                            # every tie, scale 1
            x[N - 1, Hkv, 3] = np.inf
            x[N - 1, 2 * Hkv, 5] = np.nan
            x[N - 1, 3 * Hkv - 1, D - 1] = -np.inf
        t = dev(x).to(dtype)
        k, v = t[:, Hkv:2 * Hkv], t[:, 2 * Hkv:]
        print(f"case append {name} step {step} D={D} Hkv={Hkv}", flush=True)
        rows = make_rows(ctx, new)
        mcd.mcd_cache_append(cache, rows, k[:N] if N else k, v[:N] if N else v, ws)
        for r in range(R):
            for i in range(new[r]):
                pos, tok = ctx[r] + i, starts(new)[r] + i
                for h in range(Hkv):
                    ref.put(pages[table[r, pos // 64], h], D, pos % 64, x[tok, Hkv + h],
                            x[tok, 2 * Hkv + h])
                    w[r, h, pos] = 0.0
        assert np.array_equal(cache.pages.cpu().numpy(), pages)
        assert np.array_equal(cache.weight.cpu().numpy(), w)
        kr, vr = (torch.full((N, Hkv, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
        mcd.mcd_cache_read(cache, rows, kr, vr, ws)
        want_k, want_v = np.zeros((N, Hkv, D)), np.zeros((N, Hkv, D))
        for r in range(R):
            for i in range(new[r]):
                for h in range(Hkv):
                    tok, pos = starts(new)[r] + i, ctx[r] + i
                    want_k[tok, h], want_v[tok, h] = ref.get(pages[table[r, pos // 64], h], D,
                                                             pos % 64)
        for got, want in ((kr, want_k), (vr, want_v)):
            assert np.array_equal(got.float().cpu().numpy(), rounded(want, dtype), equal_nan=True)
    assert mcd.mcd_read_device_status(ws) == 0


def test_append_with_slots_and_shared_prefix():
    """Rows write to the slots they name; slots that share a full page keep sharing it."""
    rng = np.random.default_rng(5)
    D, H = 64, 2
    cache, pages, table, _, _ = make_cache(rng, [70, 70, 100], H, D)
    table[1, 0] = table[0, 0]                                     # a Companion's copied prefix
    cache.table.copy_(i32(table))
    slot, ctx, new = [2, 0, 1], [90, 66, 64], [10, 4, 6]
    x = rounded(rng.standard_normal((20, 2 * H, D)), BF16)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    t = dev(x).to(BF16)
    mcd.mcd_cache_append(cache, make_rows(ctx, new, slot), t[:, :H], t[:, H:], ws)
    for r in range(3):
        for i in range(new[r]):
            pos, tok = ctx[r] + i, starts(new)[r] + i
            for h in range(H):
                ref.put(pages[table[slot[r], pos // 64], h], D, pos % 64, x[tok, h], x[tok, H + h])
    assert np.array_equal(cache.pages.cpu().numpy(), pages)
    assert mcd.mcd_read_device_status(ws) == 0


# ---- attention ---------------------------------------------------------------

def bounds(k, q, scale, dtype, weight, size):
    """How far out and received weight may be.  Keys, values and bf16 queries enter the products
    exactly.  A logit is a chain of D / 32 matrix instructions (three times that in fp32) over 32
    products each, and one fused multiply-add: at most c = 3 D / 32 + 6 roundings of 2^-23 of the
    sum of magnitudes.  A softmax weight is off by that and by some roundings of the exponential
    and of the sums (16 of 2^-23).  bf16: weights of 16 bits leave the output's own rounding to 8
    bits, at most 2^-8 of the output and so of the sum of p |v|."""
    D = k.shape[-1]
    finite = np.nan_to_num(np.abs(k))
    reach = scale * np.einsum("hld,nhd->nhl", finite,
                              np.abs(q).reshape(q.shape[0], k.shape[0], -1, D).max(2)).max() \
        if k.shape[1] else 0.0
    rel = 2 * (3 * D / 32 + 6) * 2.0 ** -23 * reach + 16 * 2.0 ** -23
    out = (rel + (2.0 ** -8 if dtype == BF16 else 2.0 ** -22)) * size + 1e-30
    return out, rel * weight + 2.0 ** -23 * weight + 1e-30, rel + 1e-6


ATTENDS = [
    # name, Hq, Hkv, D, dtype, context, new tokens
    ("single_position", 1, 1, 64, BF16, [0], [1]),
    ("page_ends", 4, 2, 128, BF16, [62, 63, 64, 65, 126, 127, 128], [1] * 7),
    ("page_ends_fp32", 4, 2, 128, F32, [62, 63, 64, 65, 126, 127, 128], [1] * 7),
    ("groups_of_five_fp32", 25, 5, 64, F32, [0, 1, 2, 333, 500], [1] * 5),
    ("one_head_for_all", 16, 1, 128, BF16, [10, 300], [1, 1]),
    ("group_of_17", 17, 1, 64, BF16, [200, 7], [1, 1]),
    ("group_of_40_fp32", 40, 1, 64, F32, [200, 7], [1, 1]),
    ("wide_heads", 6, 2, 256, BF16, [5, 190], [1, 1]),
    ("wide_heads_fp32", 3, 3, 256, F32, [5, 130], [1, 1]),
    ("empty_rows", 4, 2, 64, BF16, [-1, 70, -5, -2], [1, 1, 3, 4]),
    ("empty_rows_fp32", 4, 2, 64, F32, [-1, 70, -70, -2], [1, 1, 80, 4]),
    ("rows_without_tokens", 8, 2, 128, BF16, [40, 0, 90, 3], [0, 1, 0, 2]),
    ("chunks", 8, 2, 128, BF16, [0, 100, 63, 5], [70, 33, 2, 1]),
    ("chunks_fp32", 4, 2, 128, F32, [0, 100], [70, 33]),
    ("chunks_of_wide_heads", 4, 2, 256, BF16, [30, 0], [40, 97]),
    ("chunks_of_64", 10, 2, 64, BF16, [3, 0, 129], [65, 130, 64]),
    ("decode_beside_a_prompt", 12, 2, 64, BF16, [300, 0, 200, 77], [1, 150, 1, 1]),
    ("short_drafts", 8, 2, 128, BF16, [500, 130, 64], [4, 4, 3]),
    ("long_row", 2, 1, 128, BF16, [9000], [1]),
    ("long_row_fp32", 1, 1, 64, F32, [9000], [1]),
    ("long_row_chunk", 2, 1, 64, BF16, [4000], [20]),
    ("long_beside_short", 4, 1, 64, BF16, [6000, 3, 0, 700], [1, 1, 1, 1]),
]
# many rows: more pages than workgroups, rows of every length, empty rows among them
_MANY = [(37 * i * i) % 1000 if i % 11 else -1 for i in range(70)]
ATTENDS += [
    ("many_rows", 10, 5, 64, BF16, _MANY, [1] * 70),
    ("many_rows_fp32", 5, 5, 128, F32, _MANY, [1] * 70),
    ("many_rows_of_wide_heads", 8, 4, 256, BF16, _MANY, [1] * 70),
    ("many_drafts", 16, 4, 128, BF16, _MANY, [i % 4 for i in range(70)]),
    ("many_rows_beside_prompts", 8, 4, 64, F32, _MANY[:40] + [0, 64], [1] * 40 + [70, 9]),
]

# tiles of 64 and 128 query rows on both sides of the choice, chunks whose pages are
# split and joined, received weight of more tiles than a page's waves
ATTENDS += [
    ("tiles_of_64_full", 8, 2, 128, BF16, [0, 200, 61], [16, 16, 5]),
    ("tiles_of_64_one_more", 8, 2, 128, BF16, [0, 200, 61], [17, 16, 5]),
    ("tiles_of_64_fp32", 8, 2, 128, F32, [900, 0, -3], [12, 2, 7]),
    ("tiles_of_64_narrow_heads_fp32", 5, 1, 64, F32, [70, 1], [12, 9]),
    ("split_chunk_fp32", 4, 1, 128, F32, [2500], [40]),
    ("split_short_chunk", 8, 1, 128, BF16, [3900, 63], [8, 3]),
    ("many_tiles_of_weights", 8, 1, 128, BF16, [130], [300]),
    ("many_tiles_of_weights_wide_heads_fp32", 4, 1, 256, F32, [100, 3], [70, 1]),
    ("rows_just_split", 4, 1, 128, BF16, [1023, 1024, 511], [1, 1, 1]),
]


@pytest.mark.parametrize("weights", [False, True], ids=["plain", "weights"])
@pytest.mark.parametrize("name,Hq,Hkv,D,dtype,ctx,new", ATTENDS, ids=[a[0] for a in ATTENDS])
def test_attend(name, Hq, Hkv, D, dtype, ctx, new, weights):
    rng = np.random.default_rng(sum(map(ord, name)))
    R, N = len(ctx), sum(new)
    slot = rng.permutation(R)
    lengths = np.zeros(R, int)
    lengths[slot] = np.maximum(np.array(ctx) + np.array(new), 0)
    cache, pages, table, w, _ = make_cache(rng, lengths, Hkv, D, weights)
    q = rounded(rng.standard_normal((N, Hq, D)) * 2, dtype)
    rows = make_rows(ctx, new, slot, start=not (name.startswith("page_ends") and not weights))
    scale = 0.07
    wide = torch.zeros((N, Hq + 3, D), dtype=dtype, device="cuda")        # strided q and out
    wide[:, :Hq] = dev(q).to(dtype)
    out = torch.full((N, Hq + 1, D), 9.0, dtype=dtype, device="cuda")
    lse = torch.full((N, Hq), 9.0, device="cuda")
    wout = torch.full_like(cache.weight, 5.0) if weights else None
    ws = cache.workspace(rows, Hq)
    ws[256:] = 255                       # what a workspace held before does not matter
    print(f"case attend {name} weights={weights}", flush=True)
    mcd.mcd_cache_attend(cache, rows, wide[:, :Hq], out[:, :Hq], ws, scale=scale, lse=lse,
                         weight_out=wout)
    assert mcd.mcd_read_device_status(ws) == 0
    assert bool((out[:, Hq] == 9.0).all())
    got, got_lse = out[:, :Hq].double().cpu().numpy(), lse.double().cpu().numpy()
    want_w = None if w is None else np.full(w.shape, 5.0)
    for r in range(R):
        a, n, s = starts(new)[r], new[r], slot[r]
        L = max(ctx[r] + n, 0)
        k, v = slot_kv(pages, table, s, L, D)
        f32_scale = float(np.float32(scale))
        o, l, wt, size = ref.attend(k, v, q[a:a + n].astype(np.float64), ctx[r], f32_scale)
        if n == 0:
            continue
        to, tw, tl = bounds(k, q[a:a + n], f32_scale, dtype, wt, size)
        assert (np.abs(got[a:a + n] - o) <= to).all(), (r, np.abs(got[a:a + n] - o).max())
        seen = np.isfinite(l)
        assert np.array_equal(np.isneginf(got_lse[a:a + n]), ~seen)
        assert (np.abs(got_lse[a:a + n] - l)[seen] <= tl + 2.0 ** -22 * np.abs(l[seen])).all()
        if weights:
            base = w[s, :, :L].astype(np.float64)
            g = wout[s, :, :L].double().cpu().numpy()
            assert (np.abs(g - (base + wt)) <= tw + 2.0 ** -23 * (base + wt)).all()
            assert bool((wout[s, :, L:] == 5.0).all())
    # in place, and the same bits again
    if weights:
        out2 = torch.zeros_like(out)
        out2[:, Hq] = 9.0
        mcd.mcd_cache_attend(cache, rows, wide[:, :Hq], out2[:, :Hq], ws, scale=scale,
                             weight_out=cache.weight)
        assert torch.equal(out, out2)
        for s in range(R):
            assert torch.equal(cache.weight[s, :, :lengths[s]], wout[s, :, :lengths[s]]) or \
                s not in slot[np.array(new) > 0]


def test_attend_default_scale_and_a_cache_without_weights():
    """scale defaults to 1 / sqrt(D); weight_out without cache.weight starts from 0."""
    rng = np.random.default_rng(3)
    cache, pages, table, _, _ = make_cache(rng, [100], 2, 64)
    rows = make_rows([99], [1])
    q = dev(rounded(rng.standard_normal((1, 4, 64)), F32))
    out, wout = torch.zeros_like(q), torch.full((1, 2, table.shape[1] * 64), 3.0, device="cuda")
    mcd.mcd_cache_attend(cache, rows, q, out, cache.workspace(rows, 4), weight_out=wout)
    k, v = slot_kv(pages, table, 0, 100, 64)
    o, _, w, size = ref.attend(k, v, q.double().cpu().numpy(), 99, 0.125)
    to, tw, _ = bounds(k, q.cpu().numpy(), 0.125, F32, w, size)
    assert (np.abs(out.double().cpu().numpy() - o) <= to).all()
    assert (np.abs(wout[0, :, :100].double().cpu().numpy() - w) <= tw).all()
    assert bool((wout[0, :, 100:] == 3.0).all())


@pytest.mark.parametrize("n", [1, 40], ids=["decode", "chunk"])
def test_values_that_are_not_finite_reach_only_what_sees_them(n):
    """A key block (scale 255) or a value (NaN scale) that is not finite: NaN for the tokens that
    see its position, nothing for those before it and for the other head."""
    rng = np.random.default_rng(8)
    D, H, ctx = 128, 2, 80
    for part in ("key", "value"):
        cache, pages, table, _, _ = make_cache(rng, [ctx + n], H, D)
        t = (ctx + n // 2) % 64
        page = table[0, (ctx + n // 2) // 64]
        if part == "key":
            pages[page, 1, 64 * D + ((t % 16) * 4 + 2) * 4 + t // 16] = 255
        else:
            at = 66 * D + 2 * (t // 4 % 4 * 16 + t // 16 * 4 + t % 4)
            pages[page, 1, at:at + 2] = [0xC0, 0x7F]
        cache.pages.copy_(dev(pages))
        rows = make_rows([ctx], [n])
        q = dev(rng.standard_normal((n, 4, D)).astype(np.float32)).to(BF16)
        out = torch.zeros_like(q)
        mcd.mcd_cache_attend(cache, rows, q, out, cache.workspace(rows, 4))
        nan = torch.isnan(out).all(-1).cpu().numpy()
        sees = np.arange(n) >= n // 2
        assert not nan[:, :2].any()
        assert np.array_equal(nan[:, 2], sees) and np.array_equal(nan[:, 3], sees)
        assert not torch.isnan(out).any(-1).cpu().numpy()[~sees].any()


def test_extreme_logits():
    """Logits of both signs far beyond what exp holds: the largest takes all, nothing overflows."""
    D = 64
    cache = mcd.Cache.alloc(2, 1, D, 1, 2)
    cache.table.copy_(i32([[1, 0]]))
    L = 70
    k = torch.zeros((L, 1, D), device="cuda")
    k[:, 0, 0] = torch.linspace(-6, 6, L, device="cuda")
    v = torch.arange(L, device="cuda").float().view(L, 1, 1).expand(L, 1, D).contiguous()
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    mcd.mcd_cache_append(cache, make_rows([0], [L]), k, v, ws)
    for sign, at in ((1.0, L - 1), (-1.0, 0)):
        q = torch.zeros((1, 1, D), device="cuda")
        q[0, 0, 0] = sign * 1e30
        out = torch.zeros_like(q)
        mcd.mcd_cache_attend(cache, make_rows([L - 1], [1]), q, out, ws, scale=1.0)
        same = [i for i in range(L) if ref.code(float(k[i, 0, 0]), 1.0)
                == ref.code(float(k[at, 0, 0]), 1.0)]
        assert abs(float(out[0, 0, 0]) - np.mean(same)) < 1e-3 * max(np.mean(same), 1)


def test_graph_replays_and_streams():
    """A step (append, attention with splits and weights) captured once, replayed while the
    contexts advance on the device, with eager work between, against eager steps on a stream of
    its own."""
    rng = np.random.default_rng(21)
    D, Hq, H, R, steps = 64, 8, 2, 3, 5
    ctx0 = np.array([130, 900, 62])
    side = torch.cuda.Stream()
    results = []
    for graphed in (False, True):
        rng = np.random.default_rng(21)
        cache, *_ = make_cache(rng, ctx0 + steps, H, D, weights=True)
        context = i32(ctx0)
        rows = mcd.CacheRows(context, max_context=1000)
        ws = cache.workspace(rows, Hq)
        qkv = torch.zeros((R, Hq + 2 * H, D), dtype=BF16, device="cuda")
        out = torch.zeros((R, Hq, D), dtype=BF16, device="cuda")

        def step(stream=None):
            mcd.mcd_cache_append(cache, rows, qkv[:, Hq:Hq + H], qkv[:, Hq + H:], ws, stream=stream)
            mcd.mcd_cache_attend(cache, rows, qkv[:, :Hq], out, ws, weight_out=cache.weight,
                                 stream=stream)

        xs = [dev(rng.standard_normal((R, Hq + 2 * H, D)).astype(np.float32)).to(BF16)
              for _ in range(steps)]
        graph = None
        if graphed:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        outs = []
        for x in xs:
            qkv.copy_(x)
            if graphed:
                graph.replay()
            else:
                side.wait_stream(torch.cuda.current_stream())
                step(side)
                torch.cuda.current_stream().wait_stream(side)
            outs.append(out.clone())
            context.add_(1)
            torch.cuda.synchronize()
        assert mcd.mcd_read_device_status(ws) == 0
        results.append(outs + [cache.weight.clone(), cache.pages.clone()])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_offsets_beyond_32_bits():
    """Pages more than 2^32 bytes into the page array, through all four operators."""
    D, H = 128, 8
    n_pages = (5 << 30) // (H * ref.page_bytes(D))
    cache = mcd.Cache.alloc(n_pages, H, D, 2, 3, weights=True)
    cache.table.copy_(i32([[n_pages - 1, n_pages - 3, -1], [n_pages - 2, -1, -1]]))
    rng = np.random.default_rng(1)
    L = 100
    kv = dev(rng.standard_normal((L, 2 * H, D)).astype(np.float32)).to(BF16)
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    rows = mcd.CacheRows(i32([0]), start=i32([0, L]), n_tokens=L, max_tokens=L, max_context=L)
    mcd.mcd_cache_append(cache, rows, kv[:, :H], kv[:, H:], ws)
    k, v = torch.zeros((L, H, D), dtype=BF16, device="cuda"), torch.zeros((L, H, D), dtype=BF16,
                                                                          device="cuda")
    mcd.mcd_cache_read(cache, rows, k, v, ws)
    rel = float((k.float() - kv[:, :H].float()).norm() / kv[:, :H].float().norm())
    assert rel < 0.2
    q = dev(rng.standard_normal((1, H, D)).astype(np.float32)).to(BF16)
    out = torch.zeros_like(q)
    last = mcd.CacheRows(i32([L - 1]), max_context=L)
    mcd.mcd_cache_attend(cache, last, q, out, ws, weight_out=cache.weight)
    kd, vd = (x.double().cpu().numpy().transpose(1, 0, 2) for x in (k, v))
    o, _, w, size = ref.attend(kd, vd, q.double().cpu().numpy(), L - 1, D ** -0.5)
    # the values read back are rounded once more to bf16
    assert (np.abs(out.double().cpu().numpy() - o) <= 2.0 ** -7 * size).all()
    assert np.abs(cache.weight[0, :, :L].double().cpu().numpy() - w).max() < 1e-5
    to = mcd.Cache(cache.pages, cache.table[1:].contiguous(), D)
    kept, n = torch.zeros((1, H, 40), dtype=torch.int32, device="cuda"), i32([0])
    mcd.mcd_cache_evict(cache, to, i32([L]), 40, 10, kept, n, ws, L)
    assert int(n) == 40
    k2, v2 = torch.zeros((40, H, D), dtype=BF16, device="cuda"), torch.zeros((40, H, D), dtype=BF16,
                                                                            device="cuda")
    mcd.mcd_cache_read(to, mcd.CacheRows(i32([0]), start=i32([0, 40]), n_tokens=40, max_tokens=40,
                                         max_context=40), k2, v2, ws)
    idx = kept[0].long().t().unsqueeze(-1).expand(-1, -1, D)
    assert torch.equal(k2, k.gather(0, idx)) and torch.equal(v2, v.gather(0, idx))
    assert mcd.mcd_read_device_status(ws) == 0


# ---- eviction ----------------------------------------------------------------

EVICTS = [
    # name, Hkv, D, lengths, keep, recent, kind of weights
    ("one", 1, 64, [1], 1, 0, "random"),
    ("nothing_to_evict", 2, 128, [5, 0, 64], 64, 8, "random"),
    ("one_too_many", 2, 64, [65, 64, 63], 64, 64, "random"),
    ("keep_one", 3, 64, [200], 1, 0, "random"),
    ("only_recent", 2, 128, [130, 500], 100, 100, "random"),
    ("none_recent", 2, 128, [130, 500], 100, 0, "random"),
    ("odd", 5, 64, [333, 97, 1027, 100], 97, 13, "random"),
    ("all_equal", 2, 64, [300], 77, 5, "equal"),
    ("mostly_nothing", 2, 128, [2100], 1000, 50, "zeros"),
    ("special", 2, 64, [400], 150, 10, "special"),
    ("close_together", 1, 64, [3000], 1500, 1, "close"),
    ("wide_heads", 2, 256, [190, 60], 70, 20, "random"),
    ("long", 2, 64, [20000, 5], 4096, 128, "random"),
]


def some_weights(rng, kind, n):
    if kind == "equal":
        return np.full(n, 0.25, np.float32)
    w = rng.exponential(1.0, n).astype(np.float32)
    if kind == "zeros":
        w[rng.random(n) < 0.8] = 0.0
    if kind == "special":
        w = rng.choice(np.array([0.0, -0.0, np.nan, np.inf, -np.inf, 1e-45, -1.0, 1.0, 3e38],
                                np.float32), n)
    if kind == "close":
        w = (np.float32(1.0).view(np.uint32) + rng.integers(0, 40, n).astype(np.uint32)) \
            .view(np.float32)
    return w


@pytest.mark.parametrize("name,Hkv,D,lengths,keep,recent,kind", EVICTS, ids=[e[0] for e in EVICTS])
def test_evict(name, Hkv, D, lengths, keep, recent, kind):
    rng = np.random.default_rng(sum(map(ord, name)))
    R = len(lengths)
    slot = rng.permutation(R)
    by_slot = np.zeros(R, int)
    by_slot[slot] = lengths
    out_len = [min(n, keep) for n in lengths]
    spare = sum(-(-n // 64) for n in out_len)
    cache, pages, table, w, free = make_cache(rng, by_slot, Hkv, D, True, spare)
    w = np.stack([[some_weights(rng, kind, w.shape[2]) for _ in range(Hkv)] for _ in range(R)])
    cache.weight.copy_(dev(w))
    to_table = np.full((R + 1, max(-(-n // 64) for n in out_len + [1])), -1, np.int32)
    at = 0
    for r, n in enumerate(out_len):
        c = -(-n // 64)
        to_table[r, :c] = free[at:at + c]
        at += c
    to = mcd.Cache(cache.pages, i32(to_table), D,
                   torch.full((R + 1, Hkv, to_table.shape[1] * 64), 5.0, device="cuda"))
    kept = torch.full((R, Hkv, keep), 77, dtype=torch.int32, device="cuda")
    n_out = torch.full((R,), 77, dtype=torch.int32, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    print(f"case evict {name}", flush=True)
    mcd.mcd_cache_evict(cache, to, i32(lengths), keep, recent, kept, n_out, ws, max(lengths),
                        slot=i32(slot))
    assert mcd.mcd_read_device_status(ws) == 0
    assert n_out.cpu().tolist() == out_len
    after = cache.pages.cpu().numpy()
    used = table[table >= 0]
    assert np.array_equal(after[used], pages[used])               # the sources are untouched
    for r, n in enumerate(lengths):
        s, m = slot[r], out_len[r]
        k, v = slot_kv(pages, table, s, n, D)
        k2, v2 = slot_kv(after, to_table, r, m, D)
        for h in range(Hkv):
            want = ref.evict(w[s, h, :n], keep, recent)
            got = kept[r, h].cpu().numpy()
            assert np.array_equal(got[:m], want) and (got[m:] == -1).all()
            assert np.array_equal(k2[h], k[h, want], equal_nan=True)
            assert np.array_equal(v2[h], v[h, want], equal_nan=True)
            tw = to.weight[r, h].cpu().numpy()
            assert np.array_equal(tw[:m], w[s, h, want], equal_nan=True)
            assert (tw[m:] == 5.0).all()


def test_evict_copies_a_row_without_weights():
    """keep >= max_length needs no weights: a Companion's own copy of its Main row."""
    rng = np.random.default_rng(2)
    cache, pages, table, _, free = make_cache(rng, [130], 2, 64, spare=3)
    to = mcd.Cache(cache.pages, i32(free[:3][None]), 64)
    kept, n = torch.zeros((1, 2, 130), dtype=torch.int32, device="cuda"), i32([0])
    mcd.mcd_cache_evict(cache, to, i32([130]), 130, 0, kept, n,
                        torch.zeros(256, dtype=torch.uint8, device="cuda"), 130)
    after = cache.pages.cpu().numpy()
    for a, b in zip(slot_kv(after, free[:3][None], 0, 130, 64), slot_kv(pages, table, 0, 130, 64)):
        assert np.array_equal(a, b)
    assert np.array_equal(kept[0, 1].cpu().numpy(), np.arange(130)) and int(n) == 130


# ---- conditions only the device sees -------------------------------------------

def test_bad_slots_pages_and_lengths_are_reported_and_skipped():
    rng = np.random.default_rng(13)
    D, H = 64, 2
    cache, pages, table, w, free = make_cache(rng, [100, 100], H, D, True)
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    kv = dev(rng.standard_normal((8, 2 * H, D)).astype(np.float32))
    q = dev(rng.standard_normal((8, 4, D)).astype(np.float32))
    cap = table.shape[1] * 64

    def all_calls(rows, n, check=True):
        """Every call on these rows: reported each time; the pages stay what they were."""
        out = torch.full((n, 4, D), 9.0, device="cuda")
        mcd.mcd_cache_append(cache, rows, kv[:n, :H], kv[:n, H:], ws)
        assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
        ko, vo = torch.full((n, H, D), 9.0, device="cuda"), torch.full((n, H, D), 9.0, device="cuda")
        mcd.mcd_cache_read(cache, rows, ko, vo, ws)
        assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
        mcd.mcd_cache_attend(cache, rows, q[:n], out, ws, weight_out=cache.weight)
        assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
        if check:
            assert np.array_equal(cache.pages.cpu().numpy(), pages)
            assert bool((ko == 9.0).all()) and bool((vo == 9.0).all())
        return out

    for start in (True, False):
        for s in (-1, 2, 1 << 30):
            out = all_calls(make_rows([50], [1], [s], start=start), 1)
            assert bool((out == 0.0).all())
        # past the table, and past the call's own bound
        all_calls(make_rows([cap], [1], start=start, max_context=cap + 1), 1)
        all_calls(make_rows([99], [1], start=start, max_context=99), 1)
    all_calls(make_rows([2 ** 31 - 2], [3], max_context=1 << 20), 3)
    all_calls(make_rows([cap - 1], [3], max_context=cap + 2), 3, check=False)
    pages[:] = cache.pages.cpu().numpy()
    # page ids out of range
    for bad in (-1, -7, len(pages), 1 << 30):
        broken = table.copy()
        broken[0, 1] = bad
        cache.table.copy_(i32(broken))
        all_calls(make_rows([70], [1]), 1)
        all_calls(make_rows([70], [1], start=False), 1)
        all_calls(make_rows([66], [5]), 5)
        kept, n = torch.zeros((1, H, 80), dtype=torch.int32, device="cuda"), i32([0])
        to = mcd.Cache(cache.pages, i32(free[None, :2]), D)
        if bad in (-1, 1 << 30):
            mcd.mcd_cache_evict(cache, to, i32([100]), 80, 80, kept, n, ws, 100)
            assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE
            pages[:] = cache.pages.cpu().numpy()
    cache.table.copy_(i32(table))
    # starts that are not ascending, or leave the tokens
    for st in ([0, 9], [-3, 2], [5, 2], [0, 4]):
        rows = mcd.CacheRows(i32([3]), start=i32(st), n_tokens=2, max_tokens=2, max_context=50)
        out = torch.full((2, 4, D), 9.0, device="cuda")
        mcd.mcd_cache_attend(cache, rows, q[:2], out, ws)
        mcd.mcd_cache_append(cache, rows, kv[:2, :H], kv[:2, H:], ws)
        assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE, st
    # eviction: a slot, a length, a destination page
    kept, n = torch.zeros((1, H, 80), dtype=torch.int32, device="cuda"), i32([0])
    to = mcd.Cache(cache.pages, i32([[-1, -1]]), D)
    for args in ((cache, i32([100]), i32([5])), (cache, i32([-1]), None), (cache, i32([101]), None),
                 (cache, i32([100]), None)):
        mcd.mcd_cache_evict(args[0], to, args[1], 80, 8, kept, n, ws, 100, slot=args[2])
        assert mcd.mcd_read_device_status(ws) == mcd.MCD_DEV_BAD_PAGE


def test_workspace_too_small_is_refused():
    rng = np.random.default_rng(4)
    cache, *_ = make_cache(rng, [3000], 1, 64, True)
    rows = make_rows([2999], [1])
    q = torch.zeros((1, 1, 64), device="cuda")
    need = mcd.mcd_cache_workspace_bytes(cache, rows, 1)
    assert need > 512
    with pytest.raises(mcd.McdError) as e:
        mcd.mcd_cache_attend(cache, rows, q, torch.zeros_like(q),
                             torch.zeros(need - 256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == mcd.MCD_E_WORKSPACE
    assert math.isfinite(float(q.sum()))
