"""harli_sample against the 64-bit oracle.

A token is a whole number and has to be the oracle's, unless the random number lies on a border of the distribution: within 1e-9 of a
border between two tokens, where rounding of either side decides (weights are fixed point with at least 38 bits below the largest, their
sums exact), the neighbour is right too.  The log probability is off by at most half a step of fp32, plus 1e-9 for the weights."""
import math

import numpy as np
import pytest
import torch

from oracle import budget_oracle as O
from paper_2511_11729_amd import binding as hb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def sample(logits, uniform, ld=None, stream=None, **settings):
    B, V = logits.shape
    ld = ld or V
    rows = torch.full((B, ld), 1e30, device=DEV)             # what lies between the rows is larger than every logit
    rows[:, :V] = torch.from_numpy(logits).to(DEV)
    dev = {k: torch.from_numpy(np.asarray(v, np.int32 if k == "top_k" else np.float32)).to(DEV) for k, v in settings.items()}
    token = torch.full((B,), -99, dtype=torch.int32, device=DEV)
    logprob = torch.full((B,), 99.0, device=DEV)
    ws = torch.empty(hb.sample_workspace_bytes(B, V), dtype=torch.uint8, device=DEV)
    hb.sample(rows[:, :V], torch.from_numpy(np.asarray(uniform, np.float32)).to(DEV), token, logprob=logprob, workspace=ws, stream=stream, **dev)
    torch.cuda.synchronize()
    return token.cpu().numpy(), logprob.cpu().numpy()


def check(logits, uniform, ld=None, **settings):
    token, logprob = sample(logits, uniform, ld, **settings)
    uniform = np.asarray(uniform, np.float32).astype(np.float64)
    for b, row in enumerate(logits):
        kw = {k: (int(v[b]) if k == "top_k" else float(np.float32(v[b]))) for k, v in settings.items()}
        want, lp = O.sample_token(row, uniform[b], **kw)
        if token[b] != want:
            kept, weight = O.sample_kept(row, **kw)
            by = sorted(zip(kept, weight))
            total = math.fsum(w for _, w in by)
            near = {O.sample_token(row, min(max(uniform[b] + e, 0.0), 1 - 1e-16), **kw)[0] for e in (-1e-9, 1e-9)}
            assert int(token[b]) in near, (b, int(token[b]), want, kw)
            lp = math.log(dict(by)[int(token[b])] / total)
        if math.isinf(lp):
            assert logprob[b] == lp
        else:
            assert abs(logprob[b] - lp) <= 2.0 ** -24 * abs(lp) + 2e-9, (b, logprob[b], lp)
    return token


def rows(B, V, seed=0, spread=2.5):
    r = np.random.default_rng(seed)
    z = r.normal(0, spread, (B, V)).astype(np.float32)
    for b in range(B):
        z[b, r.integers(0, V, max(1, V // 50))] += np.float32(r.uniform(2, 9))
    return z, r


def mixed(B, V, r):
    return dict(temperature=r.uniform(0.3, 2.0, B), top_k=r.choice([0, 1, 2, 5, 50, V - 1, V, V + 7, -3], B),
                top_p=r.choice([1.0, 0.0, -1.0, 0.1, 0.5, 0.9, 0.999, 2.0], B), min_p=r.choice([0.0, -1.0, 0.01, 0.2, 1.0], B))


@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 255, 1000, 1023, 1025, 4097])
def test_every_filter_at_small_vocabularies(V):
    z, r = rows(24, V, V)
    check(z, r.random(24))
    for name, v in mixed(24, V, r).items():
        check(z, r.random(24), **{name: v})
    check(z, r.random(24), ld=V + 5, **mixed(24, V, r))


@pytest.mark.parametrize("V,B", [(8000, 6), (32000, 5), (50257, 3), (128256, 3), (152064, 2)])
def test_vocabularies_of_models(V, B):
    z, r = rows(B, V, V)
    check(z, r.random(B))
    check(z, r.random(B), temperature=np.full(B, 0.7), top_k=np.full(B, 40))
    check(z, r.random(B), temperature=np.full(B, 1.3), top_p=np.full(B, 0.9))
    check(z, r.random(B), min_p=np.full(B, 0.05))
    check(z, r.random(B), ld=V + 3, temperature=np.full(B, 1.0), top_k=np.full(B, 500), top_p=np.full(B, 0.95), min_p=np.full(B, 0.001))


@pytest.mark.parametrize("levels", [1, 2, 7, 40])
def test_equal_logits_go_by_index(levels):
    """Logits on a few levels: every cut falls inside a run of equal ones."""
    r = np.random.default_rng(levels)
    z = (r.integers(0, levels, (20, 3000)) / 4.0).astype(np.float32)
    z[::2] = np.where(z[::2] == 0, np.where(r.random(z[::2].shape) < 0.5, 0.0, -0.0), z[::2])
    check(z, r.random(20), top_k=r.integers(1, 3000, 20))
    check(z, r.random(20), top_p=r.random(20))
    check(z, r.random(20), top_k=r.integers(1, 3000, 20), top_p=r.random(20), temperature=r.uniform(0.1, 3, 20))
    assert np.array_equal(check(z, r.random(20), temperature=np.zeros(20)), z.argmax(1))


def test_masks_infinities_and_nan():
    z, r = rows(12, 500, 4)
    z[0] = -np.inf
    z[1, 1:] = -np.inf
    z[2, ::2] = -np.inf
    z[3] = np.finfo(np.float32).min
    z[4, 100:] = np.finfo(np.float32).min
    z[5, 7], z[5, 9] = np.inf, np.inf
    z[6, ::3] = np.nan
    z[7] = np.nan
    z[8, 3] = np.finfo(np.float32).max
    z[9, :499] = -np.inf
    z[10, 10:] = np.nan
    for seed in range(3):
        u = np.random.default_rng(seed).random(12)
        check(z, u)
        check(z, u, **mixed(12, 500, np.random.default_rng(seed + 9)))
        check(z, u, temperature=np.full(12, np.inf))
        check(z, u, temperature=np.full(12, 1e-30))
        check(z, u, temperature=np.full(12, 1e-45))
        check(z, u, top_k=np.full(12, 300), top_p=np.full(12, 0.7))
    assert check(z, r.random(12), temperature=np.full(12, np.nan))[0] == -1


@pytest.mark.parametrize("offset", [3e3, -1e6, 1e8, -3e9, 2e11, -1e15])
def test_logits_far_from_zero(offset):
    """Floats lie up to thousands of units apart out there; a temperature of their distance makes neighbours worth telling apart."""
    r = np.random.default_rng(3)
    step = float(np.spacing(np.float32(abs(offset))))
    z = (np.float32(offset) + np.float32(step) * r.integers(-6, 7, (12, 5000)).astype(np.float32)).astype(np.float32)
    z[0, ::7], z[1, ::3], z[2, 5:] = np.finfo(np.float32).min, -np.inf, np.nan
    for t in (0.03, 0.7, 5.0, step, step / 50, step * 40):
        check(z, r.random(12), temperature=np.full(12, t))
        check(z, r.random(12), temperature=np.full(12, t), top_k=np.full(12, 700), top_p=np.full(12, 0.9), min_p=np.full(12, 1e-4))


def test_largest_vocabulary():
    """2^20 tokens: spread out, and all alike (more tokens in one bin than are listed: the row itself is searched)."""
    r = np.random.default_rng(5)
    V = 1 << 20
    z = np.stack([r.normal(0, 2.5, V).astype(np.float32), np.zeros(V, np.float32)])
    check(z, [0.3, 0.7])
    check(z, [0.9, 0.2], top_k=[50, 600000])
    check(z, [0.6, 0.999], top_k=[1000, V - 1], min_p=[0.01, 0.5])
    token, logprob = sample(z, [0.5, 0.5], top_p=[0.9, 0.25])
    assert token[1] == V // 8 and logprob[1] == np.float32(-math.log(V // 4))    # half of the first quarter


@pytest.mark.parametrize("spread", [0.01, 0.3, 1.0, 20.0])
def test_flat_and_steep_rows_of_a_large_vocabulary(spread):
    """Narrow rows have more tokens in a bin than are listed, wide ones cuts below the bins."""
    z, r = rows(4, 50257, 11, spread)
    check(z, r.random(4), top_k=[10, 1000, 20000, 50000], temperature=[0.05, 1.0, 1.0, 3.0])
    check(z, r.random(4), min_p=[1e-9, 0.5, 0.9, 1e-4], temperature=[0.05, 1.0, 1.0, 3.0])


@pytest.mark.parametrize("u", [0.0, -0.0, -1.0, float("nan"), 1.0, 2.0, float("inf"), np.nextafter(np.float32(1), np.float32(0)), 1e-30, 1e-45])
def test_random_numbers_at_and_past_the_ends(u):
    z, r = rows(6, 900, 2)
    settings = mixed(6, 900, r)
    token, _ = sample(z, np.full(6, u, np.float32), **settings)
    for b in range(6):
        kept, w = O.sample_kept(z[b], **{k: (int(v[b]) if k == "top_k" else float(np.float32(v[b]))) for k, v in settings.items()})
        assert token[b] == (max(i for i, x in zip(kept, w) if x > 2.0 ** -50) if u >= 1 else O.sample_token(z[b], u, **{
            k: (int(v[b]) if k == "top_k" else float(np.float32(v[b]))) for k, v in settings.items()})[0])


def test_settings_that_are_not_a_number_are_off():
    z, r = rows(4, 700, 6)
    u = r.random(4)
    nan = np.full(4, np.nan)
    a, b = sample(z, u), sample(z, u, top_p=nan, min_p=nan)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_the_draws_follow_the_distribution():
    """4096 rows of the same logits and evenly spaced random numbers: each token is drawn as often as its share says, to one row."""
    r = np.random.default_rng(0)
    z = r.normal(0, 1.5, 37).astype(np.float32)
    n = 4096
    token, _ = sample(np.tile(z, (n, 1)), (np.arange(n) + 0.5) / n, temperature=np.full(n, 0.8), top_k=np.full(n, 20))
    kept, w = O.sample_kept(z, temperature=float(np.float32(0.8)), top_k=20)
    share = np.zeros(37)
    share[kept] = np.asarray(w) / math.fsum(w)
    assert np.all(np.abs(np.bincount(token, minlength=37) - share * n) <= 1.0 + 1e-6)


def test_the_same_row_gives_the_same_token_in_any_batch_and_captured():
    z, r = rows(40, 32000, 8)
    settings = mixed(40, 32000, r)
    u = r.random(40)
    token, logprob = sample(z, u, **settings)
    for b in range(0, 40, 7):
        t, lp = sample(z[b: b + 1], u[b: b + 1], **{k: v[b: b + 1] for k, v in settings.items()})
        assert t[0] == token[b] and lp[0] == logprob[b]
    zd, ud = torch.from_numpy(z).to(DEV), torch.from_numpy(u.astype(np.float32)).to(DEV)
    dev = {k: torch.from_numpy(np.asarray(v, np.int32 if k == "top_k" else np.float32)).to(DEV) for k, v in settings.items()}
    out, lp = torch.empty(40, dtype=torch.int32, device=DEV), torch.empty(40, device=DEV)
    ws = torch.empty(hb.sample_workspace_bytes(40, 32000), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hb.sample(zd, ud, out, logprob=lp, workspace=ws, stream=torch.cuda.current_stream(), **dev)
    for _ in range(3):
        out.fill_(-5)
        ws.fill_(0x5a)                                       # whatever is in the workspace
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), token) and np.array_equal(lp.cpu().numpy(), logprob)


def test_two_streams_with_workspaces_apart():
    z, r = rows(8, 32000, 9)
    u = r.random(8)
    want = sample(z, u, top_p=np.full(8, 0.9))
    outs = []
    zd, ud, p = torch.from_numpy(z).to(DEV), torch.from_numpy(u.astype(np.float32)).to(DEV), torch.full((8,), 0.9, device=DEV)
    torch.cuda.synchronize()
    for _ in range(2):
        st = torch.cuda.Stream()
        token, ws = torch.empty(8, dtype=torch.int32, device=DEV), torch.empty(hb.sample_workspace_bytes(8, 32000), dtype=torch.uint8, device=DEV)
        outs.append((token, ws, st))
    torch.cuda.synchronize()
    for token, ws, st in outs:
        hb.sample(zd, ud, token, top_p=p, workspace=ws, stream=st)
    torch.cuda.synchronize()
    for token, _, _ in outs:
        assert np.array_equal(token.cpu().numpy(), want[0])


# ---- top-p where a row's tokens are too many to list, against running sums over the whole row
def tokens_at(row, uniform, tol, temperature=1.0, top_k=0, top_p=1.0):
    """What the definition draws when the weight that top-p asks for is off by up to `tol` (of the largest weight's) and the random number
    by 1e-9: tokens at the borders of both."""
    z = row.astype(np.float64)
    order = np.argsort(-z, kind="stable")
    if 0 < top_k < len(z):
        order = order[:top_k]
    w = np.exp((z[order] - z[order[0]]) / temperature)
    upto = np.cumsum(w.astype(np.longdouble))
    got = set()
    for e in (-tol, 0.0, tol):
        m = len(order) if top_p >= 1 else 1 + int(np.count_nonzero(upto[:-1] < top_p * upto[-1] + e))
        index = np.sort(order[:m])
        run = np.cumsum(np.exp((z[index] - z[order[0]]) / temperature).astype(np.longdouble))
        for d in (-1e-9, 0.0, 1e-9):
            got.add(int(index[-1 if uniform >= 1 else min(int(np.searchsorted(run, max(uniform + d, 0.0) * run[-1], "right")), m - 1)]))
    return got


@pytest.mark.parametrize("level", [-8.0, -20.0, -25.0])
@pytest.mark.parametrize("V", [20000, 1 << 17, 1 << 20])
def test_top_p_inside_a_tail_of_light_tokens(level, V):
    """A heavy token and a tail that weighs little, all of it in a few bins (or below them): top-p close to 1 ends inside the tail.  The
    last token kept is drawn with a random number of 1.  Weights are off by at most 2^-51 each from rounding to fixed point and by 2^-44
    of themselves, sums of them by as much."""
    z = np.full((6, V), np.float32(level))
    z -= np.float32(np.spacing(np.float32(abs(level)))) * (np.arange(V) // 8).astype(np.float32)
    z[:, 0] = 0
    tail = np.exp(z[0, 1:].astype(np.float64)).sum()
    p = np.minimum(np.float32(1 - tail / (1 + tail) * np.array([0.9, 0.7, 0.5, 0.3, 0.1, 0.02])), np.nextafter(np.float32(1), np.float32(0)))
    token, _ = sample(z, np.ones(6), top_p=p)
    tol = V * 2.0 ** -51 + 2.0 ** -44 * (1 + tail)
    for b in range(6):
        near = tokens_at(z[b], 1.0, tol, top_p=float(p[b]))
        assert min(near) <= int(token[b]) <= max(near), (b, int(token[b]), near)


@pytest.mark.parametrize("spread", [0.01, 0.3, 1.0, 20.0])
def test_top_p_and_top_k_of_flat_and_steep_rows(spread):
    z, r = rows(6, 50257, 12, spread)
    t = np.array([0.05, 1.0, 1.0, 3.0, 1.0, 0.3], np.float32)
    k = np.array([0, 0, 20000, 50000, 1000, 45000])
    for p in (0.1, 0.9, 0.999, 1 - 2.0 ** -20, 1 - 2.0 ** -24):
        u = r.random(6).astype(np.float32)
        token, _ = sample(z, u, temperature=t, top_k=k, top_p=np.full(6, p))
        plain, _ = sample(z, u, temperature=t, top_p=np.full(6, p))
        for b in range(6):
            total = float(np.exp((z[b].astype(np.float64) - z[b].max()) / float(t[b])).sum())
            tol = 50257 * 2.0 ** -51 + 2.0 ** -43 * total
            assert int(token[b]) in tokens_at(z[b], float(u[b]), tol, float(t[b]), int(k[b]), float(np.float32(p))), (p, b)
            assert int(plain[b]) in tokens_at(z[b], float(u[b]), tol, float(t[b]), 0, float(np.float32(p))), (p, b)


def test_as_many_rows_as_a_call_takes():
    B, V = 65535, 3
    z = torch.randn(B, V, device=DEV, generator=torch.Generator(DEV).manual_seed(0))
    token, logprob = torch.empty(B + 1, dtype=torch.int32, device=DEV), torch.empty(B, device=DEV)
    token.fill_(-7)
    u = (torch.arange(B, device=DEV) + 0.5) / B
    ws = torch.empty(hb.sample_workspace_bytes(B, V), dtype=torch.uint8, device=DEV)
    hb.sample(z, u, token, logprob=logprob, workspace=ws)
    torch.cuda.synchronize()
    w = torch.exp(z.double() - z.double().amax(1, keepdim=True))
    upto = w.cumsum(1)
    share = u.double()[:, None] * upto[:, -1:]
    want = (upto <= share).sum(1).clamp(max=V - 1)
    clear = ((upto - share).abs().amin(1) > 1e-9)                # (fp32 quotients of whole numbers: some lie on a border)
    assert clear.sum() > B - 10 and torch.equal(token[:B][clear].long(), want[clear]) and int(token[B]) == -7
    lp = torch.log(w.gather(1, token[:B, None].long()) / upto[:, -1:])[:, 0]
    assert bool(((logprob.double() - lp).abs() <= 2.0 ** -24 * lp.abs() + 2e-9).all())


def test_rows_past_four_billion_logits():
    ld, V = (1 << 31) + 5, 5000
    rows_, r = rows(3, V, 14)
    big = torch.empty(2 * ld + V, device=DEV)
    z = torch.as_strided(big, (3, V), (ld, 1))
    z.copy_(torch.from_numpy(rows_))
    settings = dict(top_k=[0, 50, 0], top_p=[0.9, 1.0, 1.0], temperature=[1.0, 0.7, 0.0])
    u = r.random(3).astype(np.float32)
    token, ws = torch.empty(3, dtype=torch.int32, device=DEV), torch.empty(hb.sample_workspace_bytes(3, V), dtype=torch.uint8, device=DEV)
    dev = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device=DEV) for k, v in settings.items()}
    hb.sample(z, torch.from_numpy(u).to(DEV), token, workspace=ws, **dev)
    torch.cuda.synchronize()
    assert np.array_equal(token.cpu().numpy(), sample(rows_, u, **settings)[0])
