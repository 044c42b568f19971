"""Values that are not numbers: a call with some takes about as long as one without, and gives what the formula gives."""
import pytest

import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def fastest(call, n=4):
    """Milliseconds of the fastest of n calls, and the last one's outputs."""
    best = INF
    for _ in range(n):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        out = call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best, out


# what a call may take: its time without such values, a few times over (rows are looked at again), and a launch's jitter.
# A walk of every row over all its tokens takes a hundred times as long at these sizes.
def limit(clean):
    return 6 * clean + 1.0


@pytest.mark.parametrize("window", [None, 4096])
@pytest.mark.parametrize("what,token,bad", [("k", 0, NAN), ("k", 9000, NAN), ("v", 0, NAN), ("v", 0, INF), ("kv", 5, NAN),
                                            ("kv", 12000, INF)])
def test_a_token_of_a_long_sequence(what, token, bad, window):
    N, Hq, Hk, d = 16384, 8, 2, 64
    q, k, v = rand(1, 1, Hq, N, d), rand(2, 1, Hk, N, d), rand(3, 1, Hk, N, d)
    call = lambda: pkg.window_attn_lse(q, k, v, window=window)  # noqa: E731
    clean, (o, lse) = fastest(call)
    if "k" in what:
        k[0, 1, token] = bad
    if "v" in what:
        v[0, 1, token] = bad
    ms, (got, got_lse) = fastest(call)
    assert pkg.get_device_status() == _lib.MOA_OK
    hit = torch.zeros(Hq, N, dtype=torch.bool, device="cuda")
    hit[Hq // 2:, token:N if window is None else token + window] = True
    wrong = hit[..., None].expand(Hq, N, d)
    if "k" in what and bad == bad:    # q . k of infinite members: no number, or +-infinity, which weighs 0 or is none
        ok = torch.isfinite(got_lse[0]) | torch.isnan(got_lse[0]) | torch.isinf(got_lse[0])
        assert bool(ok.all())
    elif bad == INF:
        assert bool((got[0][wrong] == INF).all())
    else:
        assert bool(torch.isnan(got[0][wrong]).all())
    if "k" in what and bad != bad:
        assert bool((torch.isnan(got_lse[0]) == hit).all())
    # rows that share a tile of tokens with it are computed another way: to half a step of bf16 for each rounding (the weights'
    # and the output's, of values below 8)
    assert bool(((got[0].float() - o[0].float()).abs() <= 2.0 ** -8 * (o[0].float().abs() + 8))[~wrong].all())
    assert torch.equal(got[0, :Hq // 2], o[0, :Hq // 2])
    assert ms <= limit(clean), (ms, clean)


def test_all_values_of_a_step():
    """A training step that has diverged: nothing is a number, and the call takes no longer."""
    q, k, v = rand(1, 2, 8, 8192, 128), rand(2, 2, 2, 8192, 128), rand(3, 2, 2, 8192, 128)
    call = lambda: pkg.window_attn_lse(q, k, v, window=1024, sinks=4)  # noqa: E731
    clean, _ = fastest(call)
    for x in ((q, k, v), (v,)):
        keep = [y.clone() for y in x]
        for y in x:
            y.fill_(NAN)
        ms, (o, lse) = fastest(call)
        assert bool(torch.isnan(o).all()) and bool(torch.isnan(lse).all()) == (len(x) == 3)
        assert ms <= limit(clean), (len(x), ms, clean)
        for y, z in zip(x, keep):
            y.copy_(z)


@pytest.mark.parametrize("lens,N", [([60000], 1), ([8000] * 3, 2), ([1000] * 8, 1), ([5000] * 40, 3), ([30000], 200)])
@pytest.mark.parametrize("where", ["q", "k", "v"])
def test_queries_and_tokens_of_a_cache(lens, N, where):
    """Clusters, equal shares, whole and cut items."""
    Hq, Hk, d, page = 8, 2, 128, 64
    B, L = len(lens), max(lens)
    per = -(-L // page)
    pool = rand(4, B * per, Hk, page, 2 * d)
    table = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    q, ln = rand(5, B, Hq, N, d), torch.tensor(lens, dtype=torch.int32, device="cuda")
    call = lambda: pkg.kv_attn_lse(q, pool, table, ln, max_len=L)  # noqa: E731
    clean, (o, _) = fastest(call)
    if where == "q":
        q[-1, 5] = NAN
    else:
        t = L - N - 1        # the last token that all queries see
        pool[int(table[-1, t // page]), 1, t % page, 0 if where == "k" else d:d if where == "k" else 2 * d] = NAN
    ms, (got, lse) = fastest(call)
    assert pkg.get_device_status() == _lib.MOA_OK
    hit = torch.zeros(B, Hq, dtype=torch.bool, device="cuda")
    hit[-1, 5 if where == "q" else slice(4, 8)] = True
    assert bool(torch.isnan(got[hit]).all()) and torch.equal(got[~hit], o[~hit])
    assert bool(torch.isnan(lse[hit]).all()) == (where != "v") and not bool(torch.isnan(lse[~hit]).any())
    assert ms <= 6 * clean + 0.2, (ms, clean)


U = 2.0 ** -8   # half a step of bf16


def formula(q, k, v, see):
    """(o, its bound) of one head in 64 bits, infinite and NaN values of v reaching the rows that see them."""
    q, k, v = q.double(), k.double(), v.double()
    scale = q.shape[1] ** -0.5
    p = torch.nan_to_num(torch.softmax((q @ k.T * scale).masked_fill(~see, -INF), 1), nan=0.0)
    finite = torch.where(torch.isfinite(v), v, 0.0)
    o, av = p @ finite, p @ finite.abs()
    size = (q.abs() @ k.abs().T * scale).masked_fill(~see, 0).amax(1, keepdim=True)
    # scores in fp32 (2 (d + 8) 2^-24 of their terms' sum), exponentials (2^-18) and sums (2^-15), weights and output in bf16
    bound = (2 * (q.shape[1] + 8) * 2.0 ** -24 * size + 2.0 ** -18 + 2.0 ** -15 + U) * av * 1.02 + U * o.abs() * 1.02 + 1e-30
    seen = lambda what: see.double() @ what.double() > 0  # noqa: E731
    up, down, none = seen(v == INF), seen(v == -INF), seen(torch.isnan(v))
    o = torch.where(up, INF, o)
    o = torch.where(down, -INF, o)
    return torch.where(none | (up & down), NAN, o), bound


def agrees(got, want, bound):
    got = got.double()
    same = torch.where(torch.isfinite(want), (got - want).abs() <= bound, got == want)
    return bool((same | (torch.isnan(got) & torch.isnan(want))).all())


def sight(N, L, window, sinks, causal=True):
    p, j = torch.arange(L - N, L, device="cuda")[:, None], torch.arange(L, device="cuda")[None]
    see = (j <= p) if causal else (j < L) & (p == p)
    return see & ((j > p - window) | (j < sinks)) if window else see


def sprinkle(v, seed, some):
    """`some` values of [.., T, d] become infinite or NaN: single features, and whole tokens."""
    g = torch.Generator().manual_seed(seed)
    flat = v.reshape(-1, v.shape[-1])
    for n in range(some):
        t, f = int(torch.randint(flat.shape[0], (), generator=g)), int(torch.randint(flat.shape[1], (), generator=g))
        flat[t, f if n % 4 else slice(None)] = (INF, -INF, NAN)[n % 3]
    return flat.view(v.shape)


@pytest.mark.parametrize("B,Hq,Hk,N,M,dk,dv,window,sinks", [
    (1, 4, 2, 300, 300, 64, 64, 50, 3),          # clusters of a CTA
    (1, 8, 2, 40, 5000, 128, 128, 900, 200),     # clusters
    (2, 8, 2, 2500, 2500, 128, 64, 300, 5),      # two row tiles, cut items
    (2, 6, 2, 1500, 1700, 64, 128, 0, 0),        # rows that no head fills
    (1, 200, 1, 203, 190, 64, 64, 33, 2),        # two chunks of heads, queries that see nothing
    (24, 8, 8, 700, 700, 64, 64, 130, 1),        # more items than CTAs
    (1, 2, 1, 5000, 5000, 128, 128, 1, 0),       # the token itself
    (1, 16, 16, 260, 20000, 64, 64, 0, 0),       # long cut items
])
def test_values_here_and_there(B, Hq, Hk, N, M, dk, dv, window, sinks):
    q, k = rand(1, B, Hq, N, dk), rand(2, B, Hk, M, dk)
    v = sprinkle(rand(3, B, Hk, M, dv), N, 12 * B)
    o = pkg.window_attn(q, k, v, window=window or None, sinks=sinks)
    assert pkg.get_device_status() == _lib.MOA_OK
    see = sight(N, M, window, sinks)
    for b in {0, B - 1}:
        for h in range(0, Hq, max(1, Hq // 8)):
            assert agrees(o[b, h], *formula(q[b, h], k[b, h // (Hq // Hk)], v[b, h // (Hq // Hk)], see)), (b, h)


@pytest.mark.parametrize("lens,Hq,Hk,N,dk,dv,page,window,sinks,causal", [
    ([5000, 3000], 8, 2, 1, 128, 128, 16, 700, 4, True),
    ([300, 0, 17, 130], 8, 4, 5, 64, 128, 48, 0, 0, True),
    ([4000] * 30, 16, 8, 2, 128, 64, 64, 600, 130, True),
    ([3000, 900], 8, 2, 700, 64, 64, 32, 257, 3, True),
    ([3000, 900], 8, 2, 300, 128, 128, 128, 0, 0, False),
    ([20000], 4, 1, 260, 64, 64, 256, 0, 0, True),
])
def test_values_here_and_there_in_a_cache(lens, Hq, Hk, N, dk, dv, page, window, sinks, causal):
    """Junk past the ends, and pages before every window whose entries of the table are anything."""
    B, per = len(lens), -(-max(lens) // page)
    g = torch.Generator(device="cuda").manual_seed(N)
    table = torch.randperm(B * per, generator=g, device="cuda").view(B, per)
    k, v = rand(6, B, Hk, per * page, dk), sprinkle(rand(7, B, Hk, per * page, dv), N, 12 * B)
    for b, n in enumerate(lens):
        k[b, :, n:], v[b, :, n:] = NAN, NAN
    pool = torch.empty(B * per, Hk, page, dk + dv, dtype=torch.bfloat16, device="cuda")
    pool[table.flatten()] = torch.cat([k, v], -1).view(B, Hk, per, page, dk + dv).transpose(1, 2).flatten(0, 1)
    pages = table.to(torch.int32)
    if window and causal:
        for b, n in enumerate(lens):
            first = max(0, n - N - window + 1) // page      # pages before it are seen by no query, but for the sinks
            pages[b, -(-sinks // page):first] = torch.arange(first + 9, device="cuda")[-(-sinks // page):first].to(torch.int32) * 977 - 5
    q = rand(8, B, Hq, N, dk)
    o = pkg.kv_attn(q, pool, pages, torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len=max(lens), window=window or None,
                    sinks=sinks, causal=causal)
    assert pkg.get_device_status() == _lib.MOA_OK
    for b in {0, 1, B - 1} & set(range(B)):
        n = lens[b]
        if n == 0:
            assert bool((o[b] == 0).all())
            continue
        see = sight(N, n, window, sinks, causal)
        for h in range(0, Hq, max(1, Hq // 4)):
            hk = h // (Hq // Hk)
            assert agrees(o[b, h], *formula(q[b, h], k[b, hk, :n], v[b, hk, :n], see)), (b, h)


# -- gradients ----------------------------------------------------------------------------------------
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "fp32": (torch.float32, 2.0 ** -24)}


def plant(x, seed, some, whole):
    """`some` rows of x [B, H, N, d] get values that are not finite: single features, or (`whole`) all of them."""
    g = torch.Generator().manual_seed(seed)
    flat = x.view(-1, x.shape[-1])
    for n in range(some):
        r, f = int(torch.randint(flat.shape[0], (), generator=g)), int(torch.randint(x.shape[-1], (), generator=g))
        flat[r, slice(None) if whole else f] = (NAN, INF, -INF)[n % 3]


def gradients_agree(q, k, v, o, lse, do, got, window, sinks, dtype):
    """Where the formula is finite, within its bound; elsewhere not finite.  One key head: q, o, do [G, N, .], k, v [M, .]."""
    G, N, dk = q.shape
    M, dv = v.shape
    u, scale, see = TYPES[dtype][1], dk ** -0.5, sight(N, M, window, sinks)
    ub = u if dtype == "bf16" else 0.0
    k, v = k.double(), v.double()
    num = lambda x: torch.where(torch.isfinite(x), x, 0.0)  # noqa: E731
    odd = lambda x: (~torch.isfinite(x)).double()  # noqa: E731
    sums = {n: torch.zeros(M, d, dtype=torch.float64, device="cuda") for n, d in (("k", dk), ("v", dv), ("ek", dk), ("ev", dv),
                                                                                 ("bk", dk), ("bv", dv))}
    for h in range(G):
        qq, gg, oo, ll = q[h].double(), do[h].double(), o[h].double(), lse[h].double()
        base = torch.where(ll == -INF, 0.0, ll)[:, None]
        p = torch.where(see, torch.exp(qq @ k.T * scale - base), 0.0)
        ds = torch.where(see, p * (gg @ v.T - (gg * oo).sum(1, keepdim=True)), 0.0)
        badp, badds = odd(p), odd(ds)
        seen = see.double()
        fp, fds = num(p), num(ds)
        size = (num(qq).abs() @ num(k).abs().T * scale).masked_fill(~see, 0).amax(1, keepdim=True)
        w = 2 * (dk + 8) * 2.0 ** -24 * size + 2.0 ** -18 + 2.0 ** -22 * num(base).abs()
        dot = (dv + 8) * 2.0 ** -24 * (num(gg).abs() @ num(v).abs().T + (num(gg) * num(oo)).abs().sum(1, keepdim=True))
        eds = (w + ub + 2.0 ** -15) * fds.abs() + fp * dot * 1.02
        want, bound = scale * fds @ num(k), scale * (eds @ num(k).abs())
        none = (badds.sum(1, keepdim=True) + seen @ odd(k)) > 0
        ok = torch.where(none, ~torch.isfinite(got[0][h]), (got[0][h].double() - want).abs() <= 1.02 * (bound + u * want.abs()) + 1e-30)
        assert bool(ok.all()), ("dq", h, (~ok).nonzero()[:4].tolist())
        sums["k"] += scale * fds.T @ num(qq)
        sums["ek"] += scale * eds.T @ num(qq).abs()
        sums["bk"] += badds.sum(0)[:, None] + seen.T @ odd(qq)
        sums["v"] += fp.T @ num(gg)
        sums["ev"] += ((w + ub + 2.0 ** -15) * fp).T @ num(gg).abs()
        sums["bv"] += badp.sum(0)[:, None] + seen.T @ odd(gg)
    for n, x in (("k", got[1]), ("v", got[2])):
        want = sums[n]
        ok = torch.where(sums["b" + n] > 0, ~torch.isfinite(x), (x.double() - want).abs() <= 1.02 * (sums["e" + n] + u * want.abs()) + 1e-30)
        assert bool(ok.all()), ("d" + n, (~ok).nonzero()[:4].tolist())


SHAPES = [  # B, H_q, H_k, N, M, d_k, d_v, window, sinks
    (1, 4, 2, 300, 300, 64, 64, 50, 3), (1, 8, 2, 900, 900, 128, 128, 130, 5), (2, 6, 2, 400, 400, 64, 128, 0, 0),
    (1, 4, 1, 500, 1700, 128, 64, 200, 0),      # tokens that no query sees
    (1, 6, 2, 700, 430, 64, 64, 90, 2),         # queries that see nothing
    (1, 2, 2, 40, 3000, 128, 128, 0, 0),        # few rows: tokens in pieces
    (1, 2, 1, 3000, 3000, 64, 64, 260, 70),     # sinks' rows in pieces
    (1, 130, 1, 90, 90, 64, 64, 20, 0),         # chunks of heads
]


@pytest.mark.parametrize("what", ["q", "k", "v", "do", "rows", "tokens", "all"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gradients(shape, dtype, what):
    """Queries, keys, values and output gradients that are not finite reach what they see, and nothing else."""
    B, Hq, Hk, N, M, dk, dv, window, sinks = shape
    x = {n: rand(i, *s).to(TYPES[dtype][0]) for i, (n, s) in enumerate(
        dict(q=(B, Hq, N, dk), k=(B, Hk, M, dk), v=(B, Hk, M, dv), do=(B, Hq, N, dv)).items())}
    sight_ = dict(window=window or None, sinks=sinks)
    for n in dict(rows=("q", "do"), tokens=("k", "v"), all=x).get(what, (what,)):
        plant(x[n], N + len(n), 2 * B, what in ("rows", "tokens"))
    hidden = M - N - window + 1                # tokens before every window
    if window and hidden > sinks and what in ("k", "v", "tokens", "all"):
        for n in "kv":
            x[n][:, :, sinks:hidden] = NAN
    if N > M and what in ("q", "do", "rows", "all"):
        for n in ("q", "do"):
            x[n][:, :, :N - M] = NAN
    o, lse = pkg.window_attn_lse(x["q"], x["k"], x["v"], **sight_)
    got = pkg.window_attn_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], **sight_)
    again = pkg.window_attn_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], **sight_)
    assert pkg.get_device_status() == _lib.MOA_OK
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, again))
    G = Hq // Hk
    for b in range(B):
        for hk in range(Hk):
            of = lambda t: t[b, hk * G:hk * G + G]  # noqa: E731
            gradients_agree(of(x["q"]), x["k"][b, hk], x["v"][b, hk], of(o), of(lse), of(x["do"]),
                            (of(got[0]), got[1][b, hk], got[2][b, hk]), window, sinks, dtype)


@pytest.mark.parametrize("what", ["q", "k", "v", "do", "all", "one k", "one v", "one q", "one do", "padding"])
@pytest.mark.parametrize("window", [None, 1024])
def test_gradients_take_no_longer(what, window):
    """Diverged steps, single values, and padding that is anything: in about a call's time."""
    N, Hq, Hk, d = 8192, 8, 2, 128
    x = {n: rand(i, 1, h, N, d) for i, (n, h) in enumerate((("q", Hq), ("k", Hk), ("v", Hk), ("do", Hq)))}
    o, lse = pkg.window_attn_lse(x["q"], x["k"], x["v"], window=window)
    clean, _ = fastest(lambda: pkg.window_attn_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], window=window))
    if what == "padding":
        for n in x:
            x[n][:, :, 5000:] = NAN if n != "do" else 0
    elif what.startswith("one"):
        x[what[4:]][0, 1, 4000, 5] = NAN
    else:
        for n in x if what == "all" else [what]:
            x[n].fill_(NAN)
    o, lse = pkg.window_attn_lse(x["q"], x["k"], x["v"], window=window)
    ms, got = fastest(lambda: pkg.window_attn_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], window=window))
    assert pkg.get_device_status() == _lib.MOA_OK
    if what == "padding" and window:
        assert bool(torch.isfinite(got[0][:, :, :5000]).all())      # real queries see real tokens only
        assert all(bool(torch.isfinite(g[:, :, :5000 - window + 1]).all()) for g in got[1:])
    # a tile once more: each step's copies, products and exponentials one after the other, five times as long at most, beside the call itself
    assert ms <= 8 * clean + 1.0, (ms, clean)


@pytest.mark.parametrize("what", ["q", "k", "do", "rows", "tokens"])
def test_gradients_of_tokens_that_sequences_share(what):
    """bf16 on CUDA cores: one sequence's keys and values, expanded over the batch."""
    B, Hq, Hk, N, M, dk, dv, window, sinks = 2, 6, 2, 300, 420, 64, 128, 70, 3
    x = {n: rand(i, *s) for i, (n, s) in enumerate(
        dict(q=(B, Hq, N, dk), k=(1, Hk, M, dk), v=(1, Hk, M, dv), do=(B, Hq, N, dv)).items())}
    for n in dict(rows=("q", "do"), tokens=("k", "v")).get(what, (what,)):
        plant(x[n], N + len(n), 4, what in ("rows", "tokens"))
    for n in "kv":
        if what in ("k", "tokens"):
            x[n][:, :, sinks:M - N - window + 1] = NAN
        x[n] = x[n].expand(B, -1, -1, -1)
    o, lse = pkg.window_attn_lse(x["q"], x["k"], x["v"], window=window, sinks=sinks)
    got = pkg.window_attn_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], window=window, sinks=sinks)
    assert pkg.get_device_status() == _lib.MOA_OK
    G = Hq // Hk
    for b in range(B):
        for hk in range(Hk):
            of = lambda t: t[b, hk * G:hk * G + G]  # noqa: E731
            gradients_agree(of(x["q"]), x["k"][b, hk], x["v"][b, hk], of(o), of(lse), of(x["do"]),
                            (of(got[0]), got[1][b, hk], got[2][b, hk]), window, sinks, "bf16")
