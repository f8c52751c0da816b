"""Log probabilities on the GPU against their definition in 64 bits: ids exactly, numbers within
bounds that count the roundings of fp32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


def reference(x, T):
    """Of one vector in float64: log p of every id, entropy, the T first ids, and for a fp32 sum of
    e^d the bounds on log p and on the entropy in units of 2^-24.
      d = x - m and its product with log2 e are rounded once each at most, and so is log2 e itself: an
      exponent is off by 5/2 |d| units, which changes S = sum e^d by 5/2 U, U = sum e^d |d|, and U by
      5/2 W, W = sum e^d d^2.  exp2 is good to one ulp (2 units).  A sum goes through at most 32
      additions of a lane, 6 of lanes, 4 of waves and 6 of parts: with the exponential's 2, the product
      e d, and an exponential and a product for the shared shift and for the join below 60 units of
      it.
    Exponentials below the smallest normal number of fp32 are 0: V 2^-126 of S at most, and 88 times
    that of U, e d being largest there at d = -126 log 2."""
    V = len(x)
    if np.isnan(x).any() or (x == INF).any() or not (x > -INF).any():
        return np.full(V, NAN), NAN, np.zeros(0, int), np.zeros(V), 0.0
    m = x.max()
    d = x - m
    e = np.exp(d)
    first = int(x.argmax())
    S = e[:first].sum() + e[first + 1:].sum()
    fin = np.where(np.isfinite(d), d, 0.0)
    U, W = -(e * fin).sum(), (e * fin * fin).sum()
    lp = d - np.log1p(S)
    log_units = (2.5 * U + 60 * S) / (1 + S) + 2 * np.log1p(S)
    order = np.lexsort((np.arange(V), -x))[:T]
    H = np.log1p(S) + U / (1 + S)
    H_units = log_units + (2.5 * W + 60 * U) / (1 + S) + U / (1 + S) * (60 * S / (1 + S) + 4) + H
    return lp, H, order[x[order] > -INF], np.abs(fin) + log_units + np.abs(fin - np.log1p(S)), H_units


def check(x, streams, tokens, T, pad, dtype, pad_columns=0, uniform=True, row=None, entropy=True,
          misalign=0):
    """x [n][sum of streams] float32 values that dtype holds."""
    n, N = x.shape
    K, off = len(streams), np.concatenate([[0], np.cumsum(streams)])
    flat = torch.full((misalign + n * (N + pad_columns),), 1e30, dtype=dtype, device="cuda")
    t = flat[misalign:].view(n, N + pad_columns)[:, :N]
    t.copy_(torch.from_numpy(x))
    logits = t.unflatten(1, (K, N // K)) if uniform else t
    lp = torch.full((n, K), 7.0, device="cuda")
    H = torch.full((n, K), 7.0, device="cuda") if entropy else None
    ids = torch.full((n, K, T), 7, dtype=torch.int32, device="cuda") if T else None
    tops = torch.full((n, K, T), 7.0, device="cuda") if T else None
    ws = torch.zeros(mcd.mcd_logprobs_workspace_bytes(n, K, max(streams), T), dtype=torch.uint8,
                     device="cuda")
    ws[256:] = 255                                  # (only the status word is zeroed)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    print(f"case n={n} streams={streams[:3]}.. T={T} {dtype}", flush=True)
    mcd.mcd_logprobs(logits, dev(tokens), lp, ws, entropy=H, top_ids=ids, top_logprobs=tops,
                     V_stream=None if uniform else np.array(streams), pad_id=pad,
                     token_row=None if row is None else dev(row))
    status = mcd.mcd_read_device_status(ws)
    lp, H = lp.cpu().numpy(), H.cpu().numpy() if entropy else None
    bad = False
    eps, tiny = 2.0 ** -24, max(streams) * 2.0 ** -126
    for i in range(n):
        for k in range(K):
            v = x[i, off[k]:off[k + 1]].astype(np.float64)
            want, ent, order, units, H_units = reference(v, T)
            r = i if row is None else row[i]
            tok = tokens[r, k] if 0 <= r < len(tokens) else None
            if tok is not None and tok == pad:
                assert lp[i, k] == 0.0
            elif tok is None or not 0 <= tok < len(v):
                assert np.isnan(lp[i, k])
                bad = True
            else:
                same(lp[i, k], want[tok], units[tok] * eps + tiny)
            if entropy:
                same(H[i, k], ent, H_units * eps + 89 * tiny)
            if T:
                got = ids[i, k].cpu().numpy()
                assert got[:len(order)].tolist() == order.tolist() and (got[len(order):] == -1).all()
                val = tops[i, k].cpu().numpy()
                for j, o in enumerate(order):
                    same(val[j], want[o], units[o] * eps + tiny)
                rest = val[len(order):]
                assert np.isnan(rest).all() if np.isnan(ent) else (rest == -INF).all()
    assert status == (mcd.MCD_DEV_BAD_TOKEN if bad else 0)
    return lp


def same(got, want, tol):
    if np.isnan(want):
        assert np.isnan(got)
    elif np.isinf(want):
        assert got == want
    else:
        assert abs(got - want) <= tol, (got, want, tol)


def rounded(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float32)).to(dtype).float().numpy()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 257, 1023, 1024, 1025, 4095, 4096, 4097, 8191,
                               8193, 40000])
def test_sizes(V, dtype):
    rng = np.random.default_rng(V)
    n = 3
    x = rounded(rng.standard_normal((n, V)) * np.array([[0.3], [2.0], [6.0]]), dtype)
    for T in (0, 1, 5, 32):
        tokens = rng.integers(0, V, (n, 1))
        check(x, [V], tokens, T, -1, dtype, misalign=V % 3, pad_columns=V % 5)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("streams", [[4096] * 8, [1024] * 16, [2048] + [1024] * 8,
                                     [5, 1, 33, 700, 1100]], ids=lambda s: f"{len(s)}x{s[0]}")
def test_streams_pads_and_token_rows(streams, dtype):
    rng = np.random.default_rng(sum(streams))
    n, K, pad = 5, len(streams), max(streams)
    uniform = len(set(streams)) == 1
    x = rounded(rng.standard_normal((n, sum(streams))) * 3, dtype)
    tokens = np.stack([rng.integers(0, V, 2 * n) for V in streams], 1)
    tokens[1, K // 2:] = pad
    row = rng.permutation(2 * n)[:n]
    row[0] = 1
    check(x, streams, tokens, 3, pad, dtype, uniform=uniform, row=row)
    check(x, streams, tokens[:n], 0, pad, dtype, uniform=uniform, entropy=False)


@pytest.mark.parametrize("V", [50, 1000, 3000, 9000])
def test_ties(V):
    """Whole vectors of one value, and few values: more candidates than are sorted at once."""
    rng = np.random.default_rng(V)
    x = np.concatenate([np.full((1, V), -2.5), np.zeros((1, V)), rng.integers(0, 3, (2, V)),
                        np.where(rng.random((1, V)) < 0.5, -0.0, 0.0)]).astype(np.float32)
    x[3, V - 1] = 9.0
    for T in (1, 4, 32):
        for dtype in (F32, BF16):
            check(x, [V], rng.integers(0, V, (5, 1)), T, V, dtype)


@pytest.mark.parametrize("lanes,each", [(32, 2), (32, 3), (33, 3), (40, 2), (32, 4)])
def test_more_candidates_than_lanes(lanes, each):
    """Neighbouring logits in twos to fours, so that the lanes' largest leave 64 to 128 candidates."""
    rng = np.random.default_rng(lanes * each)
    x = (rng.standard_normal((6, 1024)) * 0.5).astype(np.float32)
    for i in range(6):
        for group in rng.permutation(64)[:lanes]:
            x[i, 4 * group:4 * group + each] = 10 + rng.random(each)
        x[i, 4 * group:4 * group + 4] = 9.5          # one lane's largest below all others
    for T in (16, 31, 32):
        check(x, [1024], rng.integers(0, 1024, (6, 1)), T, -1, F32)


@pytest.mark.parametrize("V", [6, 900, 5000, 9000])
def test_masked_and_not_finite(V):
    rng = np.random.default_rng(V)
    x = (rng.standard_normal((9, V)) * 2).astype(np.float32)
    x[0] = -INF                                     # nothing left
    x[1], x[1, V // 2] = -INF, 3.0                  # one id left
    x[2, 1:] = -INF
    x[3, V - V // 3:] = -INF
    x[4, V - 1] = NAN
    x[5, 0] = INF
    x[6, 1], x[6, 2] = -INF, INF
    x[7] = -INF
    x[7, V - 1] = NAN
    x[8] = torch.finfo(F32).min                     # the type's lowest value is a number
    tokens = np.full((9, 1), V // 2)
    for T in (0, 5, 32):
        check(x, [V], tokens, T, -1, F32)
    tokens[3], tokens[8] = V - 1, 0                 # a masked token
    check(x, [V], tokens, 2, -1, F32)


def test_nearly_certain_and_large():
    """log p of a token that is nearly certain is small and keeps its digits; logits near the
    largest of fp32 do not overflow."""
    V = 5000
    x = np.zeros((4, V), np.float32)
    x[0, 4321] = 30.0
    x[1, 17] = 88.0
    x[2] = np.linspace(-3e38, 3e38, V)
    x[3, 5], x[3, 4900] = 40.0, 40.0
    lp = check(x, [V], np.array([[4321], [17], [V - 1], [5]]), 3, -1, F32)
    assert lp[0, 0] == pytest.approx(-np.log1p(4999 * np.exp(-30.0)), rel=1e-5) and lp[0, 0] != 0
    assert abs(lp[1, 0] + 4999 * np.exp(-88.0)) < 5000 * 2.0 ** -126 and lp[2, 0] == 0.0
    assert lp[3, 0] == pytest.approx(-np.log(2), rel=1e-6)


def test_bad_tokens():
    x = np.random.default_rng(0).standard_normal((4, 2 * 10)).astype(np.float32)
    tokens = np.array([[0, 9], [-1, 3], [10, 11], [5, 12]])
    check(x, [10, 10], tokens, 2, 12, F32)
    check(x, [10, 10], tokens[:1], 0, 12, F32, row=np.array([0, 1, -1, 7]))


def test_many_rows_large_vocabulary():
    """Parts of 8192 logits (more than 2048 parts of 4096)."""
    rng = np.random.default_rng(9)
    n, V = 70, 151936
    x = rounded(rng.standard_normal((n, V)).astype(np.float32) * 2, BF16)
    x[0, V - 5000:] = -INF
    check(x, [V], rng.integers(0, V - 5000, (n, 1)), 32, -1, BF16)


def test_longest_vector_and_refusal():
    rng = np.random.default_rng(3)
    V = 1 << 19
    x = (rng.standard_normal((1, V)) * 2).astype(np.float32)
    check(x, [V], np.array([[V - 1]]), 32, -1, F32)
    with pytest.raises(mcd.McdError):
        mcd.mcd_logprobs_workspace_bytes(1, 1, V + 1, 0)


def test_captured_and_replayed():
    """A graph of two calls that share a workspace, replayed with new logits."""
    gen = torch.Generator("cuda").manual_seed(0)
    x = torch.randn((6, 1, 20000), generator=gen, device="cuda")
    y = torch.randn((9, 4, 700), generator=gen, device="cuda")
    tx = torch.zeros((6, 1), dtype=torch.int32, device="cuda")
    ty = torch.full((9, 4), 3, dtype=torch.int32, device="cuda")
    ws = torch.zeros(mcd.mcd_logprobs_workspace_bytes(9, 4, 20000, 4), dtype=torch.uint8,
                     device="cuda")
    out = [torch.zeros(s, device="cuda") for s in ((6, 1), (6, 1), (6, 1, 4), (9, 4))]
    ids = torch.zeros((6, 1, 4), dtype=torch.int32, device="cuda")

    def calls():
        mcd.mcd_logprobs(x, tx, out[0], ws, entropy=out[1], top_ids=ids, top_logprobs=out[2])
        mcd.mcd_logprobs(y, ty, out[3], ws)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        x.normal_(generator=gen)
        y.normal_(generator=gen)
        graph.replay()
        got = [t.clone() for t in out + [ids]]
        calls()
        for a, b in zip(got, out + [ids]):
            assert torch.equal(a, b)
    assert mcd.mcd_read_device_status(ws) == 0


def test_another_stream():
    side = torch.cuda.Stream()
    x = torch.randn((4, 2, 3000), device="cuda")
    tok = torch.ones((4, 2), dtype=torch.int32, device="cuda")
    lp = torch.zeros((4, 2), device="cuda")
    ws = torch.zeros(mcd.mcd_logprobs_workspace_bytes(4, 2, 3000, 0), dtype=torch.uint8,
                     device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    mcd.mcd_logprobs(x, tok, lp, ws, stream=side.cuda_stream)
    side.synchronize()
    want = torch.log_softmax(x.double(), 2)[:, :, 1]
    # |log p| below 16 here: its own rounding and 60 units of the sum (see reference)
    assert (lp - want).abs().max() <= 2.0 ** -24 * (16 + 60 + 2.5 * 16)


def heads_of_any_size(rng, V, dtype):
    """Vectors whose largest logit is every power of two from 2^10 on, times three mantissas and of
    both signs, with logits close below it and far from it."""
    rows = []
    for e in range(10, 128):
        for mantissa in (1.0, 1.372, 1.9):
            for sign in (1.0, -1.0):
                m = sign * mantissa * 2.0 ** e
                if sign > 0:
                    x = rng.standard_normal(V) * 4
                else:
                    x = np.maximum(m * (1 + rng.random(V)), torch.finfo(F32).min)
                near = rng.permutation(V)[:min(V, 9)]
                x[near] = m - abs(m) * 2.0 ** -rng.integers(4, 25, len(near))
                x[near[0]] = m
                rows.append(x)
    lowest = torch.finfo(dtype).min
    return np.stack([rounded(np.maximum(x, lowest), dtype) for x in rows])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 900, 3000, 9000])
def test_largest_logits_of_any_size(V, dtype):
    """Logits in the thousands (drawn at a small temperature) up to the types' largest: a
    distribution all the same, in one wave, in four and in parts that are joined."""
    rng = np.random.default_rng(V)
    x = heads_of_any_size(rng, V, dtype)
    tokens = np.where(rng.random(len(x)) < 0.5, x.argmax(1), rng.integers(0, V, len(x)))[:, None]
    for T in (0, 1, 5):
        check(x, [V], tokens, T, -1, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V,n", [(9000, 1), (20000, 500)])
def test_parts_of_masked_logits(V, n, dtype):
    """A mask of a finite value that covers whole parts of a vector beside ordinary logits, in parts of
    4096 and (more than 2048 of those) of 8192 logits."""
    rng = np.random.default_rng(n)
    fills = [-1e4, -1e9, -1e10, -1e12, -1e15, -1e20, -1e25, -1e30, -1e36, torch.finfo(dtype).min]
    x = rng.standard_normal((max(n, len(fills)), V)) * 2
    for i in range(len(x)):
        part = 8192 if n > 1 else 4096
        kept = slice(0, part) if i % 2 else slice(part, 2 * part)
        masked = np.ones(V, bool)
        masked[kept] = False
        x[i, masked] = fills[i % len(fills)]
    x = rounded(x, dtype)
    tokens = rng.integers(0, V, (len(x), 1))
    for T in (0, 1, 5):
        check(x, [V], tokens, T, -1, dtype)


def test_as_many_vectors_as_a_launch_takes():
    """2^26 - 4 vectors: 2^24 - 1 workgroups."""
    n = (1 << 26) - 4
    x = torch.randn((n, 1, 2), dtype=BF16, device="cuda")
    tokens = torch.randint(0, 2, (n, 1), dtype=torch.int32, device="cuda")
    lp = torch.full((n, 1), 7.0, device="cuda")
    ws = torch.zeros(mcd.mcd_logprobs_workspace_bytes(n, 1, 2, 0), dtype=torch.uint8, device="cuda")
    mcd.mcd_logprobs(x, tokens, lp, ws)
    assert mcd.mcd_read_device_status(ws) == 0
    for part in (slice(0, 1 << 20), slice(n // 2, n // 2 + (1 << 20)), slice(n - (1 << 20), n)):
        want = torch.log_softmax(x[part].double(), 2).gather(2, tokens[part, :, None].long())[..., 0]
        # |log p| below 16 and 60 units of the sum (see reference)
        assert (lp[part] - want).abs().max() <= 2.0 ** -24 * (16 + 60 + 2.5 * 16)
    assert bool((lp <= 0).all())
