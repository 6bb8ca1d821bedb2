"""Vocabulary head without kept logits: forward and backward against the 64-bit oracle."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import DTYPES, HALF, TINY, Guarded, close, np64, rnd
from oracle import psattn_block_oracle as blk
from oracle import psattn_oracle as orc

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24

# offset, prompt lengths, response pointers, response lengths, tokens in all
TABLES = {
    "one_token": ([0], [1], [0, 1], [1], 2),
    "two_responses": ([0], [5], [0, 2], [4, 6], 15),
    "empty_responses_and_prompts": ([1, 20, 33], [4, 0, 3], [0, 3, 5, 5], [2, 0, 5, 3, 6], 40),
    "three_samples": ([0, 40, 90], [10, 7, 30], [0, 2, 4, 6], [12, 9, 20, 21, 3, 1], 130),
    "many_responses": ([0], [9], [0, 12], [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 1, 1], 70),
    "sixty_five_items": ([3], [8], [0, 1], [65], 90),
    "packed": ([0, 300], [100, 20], [0, 2, 4], [60, 70, 40, 90], 460),
    "long": ([0], [5], [0, 2], [300, 420], 740),
}
MORE = {
    "halfway": ([3 * i for i in range(40)], [1] * 40, list(range(41)), [1] * 40, 120),
    "again": ([0], [1], [0, 2], [1300, 1300], 2604),
}


def _inputs(table, V, h, dtype, seed=0, lean=4.0):
    off, P, ptr, rl, T = {**TABLES, **MORE}[table]
    rng = np.random.default_rng(V * 31 + h + seed)
    W = rnd(rng, V, h, scale=1.3 * h ** -0.5, dtype=dtype)
    ids = rng.integers(0, V, T)
    items = orc.prediction_items(off, P, ptr, rl)
    X = rng.standard_normal((T, h))
    for _, r, t in items:
        X[r] = X[r] + W[ids[t]] * rng.uniform(0, lean)
    X = torch.from_numpy(X).to(DTYPES[dtype]).double().numpy()
    d = torch.from_numpy(rng.standard_normal(len(rl))).float().double().numpy()
    return X, W, ids, items, d


def _call(table, X, W, ids, d, dtype, shift=0):
    off, P, ptr, rl, T = {**TABLES, **MORE}[table]
    plan = ps.LogprobPlan(off, P, ptr, rl, T)
    dev = Guarded(dtype, shift)
    tX, tW = dev.put(X), dev.put(W)
    tid = dev.put(np.asarray(ids, dtype=np.int32), dtype=torch.int32)
    f32 = torch.float32
    lse, logp = dev.empty(T, dtype=f32), dev.empty(len(rl), dtype=f32)
    lse.fill_(7.0)
    ps.psattn_head_logprob_fwd(plan, tX, tW, tid, row_lse=lse, resp_logp=logp)
    dX, dW = ps.psattn_head_logprob_bwd(plan, tX, tW, tid, lse, dev.put(d, dtype=f32), dX=dev.empty(*X.shape), dW=dev.empty(*W.shape))
    dev.check()
    return lse, logp, dX, dW


def _check(X, W, ids, items, d, got, dtype):
    """Error bounds.  A logit is a sum of h products: (h + 2) roundings of the magnitudes' sum.  exp(z - ref), by the hardware's exp2 or the
    library's: |z - ref| 2^-23 + 2^-22 relatively, on top of its argument's error; the sum over the vocabulary runs in chains of
    at most V / 64 + 100 additions and joins.  A gradient of a logit is d (1[.] - p), rounded to the element type."""
    lse, logp, dX, dW = got
    V, h = W.shape
    half = HALF[dtype]
    rows = sorted({r for _, r, _ in items})
    Z = X @ W.T
    ez = (h + 2) * EPS32 * (np.abs(X) @ np.abs(W.T))
    ref, per = blk.head(X, W, ids, items)
    P = np.exp(Z - ref[:, None])
    far = np.abs(Z - ref[:, None])
    e_lse = (P * (ez + EPS32 * (2 * far + 8))).sum(1) + ez.max(1) * 1e-3 + (V / 64 + 100) * EPS32 + 4 * EPS32 * np.abs(ref)
    g = np64(lse)
    close(g[rows], ref[rows], e_lse[rows], "row_lse")
    quiet = np.setdiff1d(np.arange(len(g)), rows)
    assert np.all(g[quiet] == 7.0), "rows that predict nothing are left alone"
    n_resp = logp.shape[0]
    want, tol, size, count = np.zeros(n_resp), np.zeros(n_resp), np.zeros(n_resp), np.zeros(n_resp)
    for (j, r, t), l in zip(items, per):
        if 0 <= ids[t] < V:
            want[j] += l
            tol[j] += e_lse[r] + ez[r, ids[t]] + 3 * EPS32 * (np.abs(Z[r]).max() + abs(l))
            size[j] += abs(l)
            count[j] += 1
    close(logp, want, tol + (count + 2) * EPS32 * size, "resp_logp")
    rX, rW, G = blk.head_grad(X, W, ids, items, d)
    # per item, as the kernels have them (rows of several items add up behind the products)
    eG, aG = np.zeros_like(G), np.zeros_like(G)
    for j, r, t in items:
        if not 0 <= ids[t] < V:
            continue
        hot = (np.arange(V) == ids[t]).astype(np.float64)
        one = abs(d[j]) * np.abs(hot - P[r])
        e = abs(d[j]) * (P[r] * (ez[r] + e_lse[r] + EPS32 * (2 * far[r] + 8)) + 2 * EPS32 * hot) + 2 * EPS32 * one + TINY
        eG[r] += e + half * (one + e)
        aG[r] += one
    close(dX, rX, half * np.abs(rX) + (1 + half) * (eG @ np.abs(W) + (V + 70) * EPS32 * (aG @ np.abs(W))) + TINY, "dX")
    close(dW, rW, half * np.abs(rW) + (1 + half) * (eG.T @ np.abs(X) + (len(items) + 4) * EPS32 * (aG.T @ np.abs(X))) + TINY, "dW")
    assert np.all(np64(dX)[quiet] == 0), "rows that predict nothing"


SIZES = [(1, 1), (2, 3), (7, 8), (64, 64), (100, 40), (127, 65), (128, 128), (129, 96), (257, 72), (300, 33), (513, 264), (1000, 129), (2049, 128), (3001, 64), (40, 1024), (31, 2047)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,h", SIZES)
def test_sizes(V, h, dtype):
    for table in ("two_responses", "packed") if V * h < 40000 else ("three_samples",):
        a = _inputs(table, V, h, dtype)
        _check(*a, _call(table, *a[:3], a[4], dtype), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("table", sorted(TABLES))
def test_tables(table, dtype):
    a = _inputs(table, 333, 104, dtype)
    _check(*a, _call(table, *a[:3], a[4], dtype), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("table,V,h", [("two_responses", 300, 64), ("packed", 130, 72), ("long", 520, 256)])
def test_unaligned(table, V, h, dtype):
    a = _inputs(table, V, h, dtype)
    _check(*a, _call(table, *a[:3], a[4], dtype, shift=1), dtype)


def test_ids_outside_the_vocabulary_give_nothing():
    X, W, ids, items, d = _inputs("packed", 200, 64, "bf16")
    for k, t in enumerate([items[0][2], items[3][2], items[-1][2]]):
        ids[t] = (-1, 200, 2 ** 31 - 1)[k]
    _check(X, W, ids, items, d, _call("packed", X, W, ids, d, "bf16"), "bf16")


def test_all_ids_outside():
    X, W, ids, items, d = _inputs("two_responses", 50, 64, "f32")
    lse, logp, dX, dW = _call("two_responses", X, W, np.full_like(ids, -5), d, "f32")
    assert torch.all(logp == 0) and torch.all(dX == 0) and torch.all(dW == 0) and torch.all(torch.isfinite(lse))


def test_nothing_predicted():
    plan = ps.LogprobPlan([0, 6], [4, 3], [0, 0, 0], [], 10)
    X, W, ids = torch.randn(10, 32, device="cuda"), torch.randn(20, 32, device="cuda"), torch.zeros(10, dtype=torch.int32, device="cuda")
    lse, logp = ps.psattn_head_logprob_fwd(plan, X, W, ids)
    dX, dW = torch.full_like(X, float("nan")), torch.full_like(W, float("nan"))
    ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, logp, dX=dX, dW=dW)
    assert logp.numel() == 0 and torch.all(dX == 0) and torch.all(dW == 0)
    empty = ps.LogprobPlan([0], [3], [0, 2], [0, 0], 5)  # responses without tokens
    lse, logp = ps.psattn_head_logprob_fwd(empty, X[:5], W, ids[:5])
    assert torch.all(logp == 0) and torch.all(lse == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_almost_certain_tokens_keep_their_log_probability(dtype):
    """A logit far above the others: log pi is -log(1 + what is left), as the sum gives it and not as a difference of large numbers."""
    T, V, h = 2, 130, 64
    W = np.zeros((V, h))
    W[:, 0] = -4.0
    W[17, 0] = 2.0
    X = np.zeros((T, h))
    X[0, 0] = 2.0
    table = TABLES["one_token"]
    ids = np.array([0, 17])
    lse, logp, dX, dW = _call("one_token", X, W, ids, np.array([1.0]), dtype)
    want = -np.log1p((V - 1) * np.exp(-12.0))
    # The sum, 1 + 8e-4, is rounded where something is added to the 1: four times in its block of 16, once per block and for the other
    # half-wave, three times over the waves, once over the tiles; then its logarithm's roundings.  16 of 2^-24 at most.
    assert abs(float(logp[0]) - want) <= 16 * EPS32 + 2.0 ** -20 * abs(want), (float(logp[0]), want)


@pytest.mark.parametrize("V", [300, 3000])
def test_not_finite_reaches_its_own_rows(V):
    """inf and NaN in rows that predict nothing, and in rows whose token is outside the vocabulary, reach nothing at all; in a row that
    predicts, its own response, its own row and dW."""
    X, W, ids, items, d = _inputs("packed", V, 64, "bf16")
    quiet = sorted(set(range(460)) - {r for _, r, _ in items})
    ids[items[5][2]] = -1
    want = _call("packed", X, W, ids, d, "bf16")
    bad = X.copy()
    bad[quiet[::2]], bad[quiet[1::2]] = np.nan, np.inf
    got = _call("packed", bad, W, ids, d, "bf16")
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    bad[items[5][1]] = np.nan
    got = _call("packed", bad, W, ids, d, "bf16")
    assert all(torch.equal(a, b) for a, b in zip(want[1:], got[1:]))  # row_lse of that row is NaN
    bad[items[20][1]] = np.nan
    got = _call("packed", bad, W, ids, d, "bf16")
    j = items[20][0]
    assert torch.isnan(got[1][j]) and torch.equal(torch.cat([got[1][:j], got[1][j + 1:]]), torch.cat([want[1][:j], want[1][j + 1:]]))
    keep = torch.ones(460, dtype=torch.bool, device="cuda")
    keep[items[20][1]] = False
    assert torch.equal(got[2][keep], want[2][keep]) and torch.isnan(got[2][~keep]).all()


def test_weight_zero_and_repeated_calls():
    X, W, ids, items, d = _inputs("packed", 500, 64, "bf16")
    first = _call("packed", X, W, ids, d, "bf16")
    again = _call("packed", X, W, ids, d, "bf16")
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    _, _, dX, dW = _call("packed", X, W, ids, np.zeros_like(d), "bf16")
    assert torch.all(dX == 0) and torch.all(dW == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_against_the_head_on_logits(dtype):
    """fp32 logits from 64-bit sums through psattn_logprob_*: the two heads agree within what their logits may differ."""
    X, W, ids, items, d = _inputs("three_samples", 700, 96, dtype)
    off, P, ptr, rl, T = TABLES["three_samples"]
    lse, logp, _, _ = _call("three_samples", X, W, ids, d, dtype)
    plan = ps.LogprobPlan(off, P, ptr, rl, T)
    lg = torch.from_numpy(X @ W.T).float().cuda()
    other, olp = ps.psattn_logprob_fwd(plan, lg, torch.from_numpy(ids.astype(np.int32)).cuda())
    rows = sorted({r for _, r, _ in items})
    ez = (98 * EPS32 * (np.abs(X) @ np.abs(W.T))).max(1) + 400 * EPS32
    assert np.all(np.abs(np64(lse) - np64(other))[rows] <= 2 * ez[rows])
    per = np.zeros(len(rl))
    for j, r, _ in items:
        per[j] += 4 * ez[r]
    assert np.all(np.abs(np64(logp) - np64(olp)) <= per + 40 * EPS32 * np.abs(np64(olp)))


def test_several_pieces_of_the_vocabulary():
    """More items than a piece has room for: 6 000 items of 60 000 tokens are 720 MB of bf16.  A strip of dW and some rows of dX against 64 bits."""
    T, V, h, P = 6001, 60000, 64, 1
    rng = np.random.default_rng(3)
    plan = ps.LogprobPlan([0], [P], [0, 1], [T - P], T)
    g = torch.Generator(device="cuda").manual_seed(3)
    X, W = torch.randn(T, h, generator=g, device="cuda").bfloat16(), (torch.randn(V, h, generator=g, device="cuda") * 0.2).bfloat16()
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    lse, logp = ps.psattn_head_logprob_fwd(plan, X, W, ids)
    d = torch.tensor([0.5], device="cuda")
    dX, dW = ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, d)
    x, w = X.double(), W.double()
    Z = x[:-1] @ w.T
    ref = torch.logsumexp(Z, 1)
    ez = (66 * EPS32 * (x[:-1].abs() @ w.abs().T)).max().item()
    assert (lse[:-1] - ref).abs().max().item() <= ez + (V / 64 + 100) * EPS32 + 2.0 ** -19
    G = torch.exp(Z.sub_(ref[:, None])).mul_(-0.5)
    G[torch.arange(T - 1, device="cuda"), ids[1:].long()] += 0.5
    a = G.abs()
    e = HALF["bf16"] * 1.01 + 4 * ez
    for got, want, size in ((dX[:-1], G @ w, a @ w.abs()), (dW, G.T @ x[:-1], a.T @ x[:-1].abs())):
        off = (got.double() - want).abs() - (HALF["bf16"] * want.abs() + (e + 6100 * EPS32) * size)
        assert off.max().item() <= 0, off.max().item()
    assert torch.all(dX[-1] == 0)


# logits in parts of k: few columns of wide rows, one row and many, with whole and odd rows
PARTS = [("one_token", 130, 4096), ("two_responses", 1000, 2056), ("three_samples", 700, 3001), ("sixty_five_items", 513, 2048), ("packed", 260, 4104), ("long", 300, 2050),
         ("empty_responses_and_prompts", 3, 5000), ("many_responses", 1, 8192)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("table,V,h", PARTS)
def test_wide_rows_of_a_small_vocabulary(table, V, h, dtype):
    a = _inputs(table, V, h, dtype)
    _check(*a, _call(table, *a[:3], a[4], dtype), dtype)


def test_few_items_have_gradients_as_exact_as_their_rounding():
    """bf16: one token.  Its gradients are one number times a row, and of that number two roundings are kept, 2^-17 of it off at most."""
    X, W, ids, items, d = _inputs("one_token", 400, 256, "bf16", lean=0.0)
    lse, logp, dX, dW = _call("one_token", X, W, ids, d, "bf16")
    rX, rW, G = blk.head_grad(X, W, ids, items, d)
    r = items[0][1]
    ez = (258 * EPS32 * (np.abs(X[r]) @ np.abs(W.T))).max() + 500 * EPS32  # of a logit and of the log-sum-exp
    rel = 2 * ez + 2.0 ** -17 + 8 * EPS32
    close(dW, rW, (HALF["bf16"] + rel) * np.abs(rW) + 2 * EPS32 * np.abs(rW) + abs(d[0]) * ez * np.abs(X[r]) + TINY, "dW")
    close(dX, rX, HALF["bf16"] * np.abs(rX) + (rel + 500 * EPS32) * (np.abs(G) @ np.abs(W)) + TINY, "dX")


@pytest.mark.parametrize("same", [False, True])
@pytest.mark.parametrize("V,h", [(1500, 512), (700, 1023)])
def test_dz_at_the_token_is_not_rounded(V, h, same):
    """More than 32 items of bf16, whose dz at their tokens lie half way between two numbers of the type: rounded, they would put the
    gradients off by 2^-8 at once.  They are off by their own rounding, e0 of the exact gradient (which moves by no more than its
    argument does: twice that in all), by what rounds dz elsewhere, of which sum_c a_c W_c has at most |a| sigma(W), and at a token's row
    by the rounding of the products' part of it."""
    n, half = 40, HALF["bf16"]
    rng = np.random.default_rng(V + h)
    W = rnd(rng, V, h, scale=h ** -0.5, dtype="bf16")
    ids = np.full(3 * n, 17) if same else np.resize(rng.permutation(V), 3 * n)
    X = rnd(rng, 3 * n, h, dtype="bf16") * (rng.permuted(np.arange(3 * n * h).reshape(3 * n, h) % h, axis=1) < 16)  # 16 terms to a logit
    items = orc.prediction_items(*MORE["halfway"][:4])
    assert len(items) == n
    ref, _ = blk.head(X, W, ids, items)
    rows, tok = np.array([r for _, r, _ in items]), np.array([ids[t] for _, _, t in items])
    P = np.exp(X @ W.T - ref[:, None])
    d = (1 + 2.0 ** -8) / (1 - P[rows, tok])
    d = torch.from_numpy(d).float().double().numpy()
    rX, rW, G = blk.head_grad(X, W, ids, items, d)
    _, _, dX, dW = _call("halfway", X, W, ids, d, "bf16")
    G, x = G[rows], X[rows]
    off = G.copy()
    off[np.arange(n), tok] = 0
    norm = np.linalg.norm
    bf = lambda a: torch.from_numpy(a).bfloat16().double().numpy()
    ez = (16 + 2) * EPS32 * (np.abs(x) @ np.abs(W.T))
    e32 = np.abs(G) * (2 * ez.max() + EPS32 * (V / 64 + 140))
    at_row = np.zeros_like(rW)
    at_row[tok] = (off.T @ x)[tok]
    for got, want, move, lost in (
            (dX, rX, half * norm(off) * norm(W, 2) + norm(e32 @ np.abs(W) + (V + 70) * EPS32 * np.abs(G) @ np.abs(W)), norm(W[tok])),
            (dW, rW, half * norm(off) * norm(x, 2) + half * norm(at_row) + norm(e32.T @ np.abs(x) + (n + 4) * EPS32 * np.abs(G).T @ np.abs(x)),
             norm(x.sum(0)) if same else norm(x))):
        bound = norm(bf(want) - want) + 2 * move
        assert bound < (norm(bf(want) - want) ** 2 + (0.99 * half * lost) ** 2) ** 0.5, "the bound tells the two apart"
        assert norm(np64(got) - want) <= bound


@pytest.mark.parametrize("V,h", [(5, 64), (400, 130), (20000, 64)])
def test_tokens_that_come_again(V, h):
    """Rows of dW that sum over items of several thousands, next to others of a single one"""
    a = _inputs("again", V, h, "bf16")
    _check(*a, _call("again", *a[:3], a[4], "bf16"), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,h", [(5, 64), (257, 72), (300, 33), (700, 256), (513, 1001)])
def test_many_items_of_a_small_vocabulary(V, h, dtype):
    """dW, of few tiles, in parts of the items"""
    a = _inputs("again", V, h, dtype)
    _check(*a, _call("again", *a[:3], a[4], dtype, 1 if h == 256 else 0), dtype)
