"""The operators around the head's logits on the GPU, against plain 64-bit
numpy: the int8 head (bitwise), sampling (tokens and counts equal), the
distillation loss and its gradient (the formula's, and differences')."""
import numpy as np
import pytest

from paper_2608_27460_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

INF = float("inf")
F32, BF16 = torch.float32, torch.bfloat16
LOWEST = {F32: torch.finfo(F32).min, BF16: torch.finfo(BF16).min}


@pytest.fixture(scope="module")
def vie():
    assert torch.cuda.is_available(), "the gpu tests need an MI355X"
    from paper_2608_27460_amd import vie as v
    return v


def say(*a):
    print(*a, flush=True)


def strided(t, ld, offset=0, fill=77.0):
    """The matrix t on the device with row stride ld, `offset` elements into its buffer; and that buffer."""
    R, V = t.shape
    buf = torch.full((offset + R * ld + 8,), fill, dtype=t.dtype, device="cuda")
    view = buf[offset:offset + R * ld].view(R, ld)[:, :V]
    view.copy_(t)
    return view, buf


def between(buf, R, V, ld, offset):
    """What lies in the buffer outside the matrix."""
    b = buf.clone()
    b[offset:offset + R * ld].view(R, ld)[:, :V] = 77.0
    return b


# ------------------------------------------------------------------ int8 head

def int8_reference(q, scale, h, out):
    """The definition, with numpy's fp32 products (rounded to nearest even)."""
    h = h.float().numpy()
    with np.errstate(invalid="ignore", divide="ignore"):
        xs = (np.abs(h).max(1) / np.float32(127)).astype(np.float32)
        bad = ~np.isfinite(h).all(1)
        x = np.where(xs[:, None] > 0, np.rint((h / np.where(xs > 0, xs, 1)[:, None]).astype(np.float32)), 0)
        x = np.clip(np.where(bad[:, None], 0, x), -127, 127)
    xs = np.where(bad, np.float32(np.nan), xs)
    z = (x.astype(np.float64) @ q.numpy().astype(np.float64).T).astype(np.float32)
    z = (z * scale.numpy()[None]).astype(np.float32)
    return torch.from_numpy((z * xs[:, None]).astype(np.float32)).to(out)


def int8_inputs(V, d, B, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(-127, 128, (V, d), generator=g, dtype=torch.int32).to(torch.int8)
    scale = torch.rand(V, generator=g) * 1e-2
    h = torch.randn(B, d, generator=g)
    h[0, 0] = 9.0
    if B > 2:
        h[1] = 0.0
    return q, scale, h.to(dtype)


def same_bits(a, b):
    a, b = a.cpu(), b.cpu()
    assert a.dtype == b.dtype and a.shape == b.shape
    i = torch.int32 if a.dtype == F32 else torch.int16
    nan = torch.isnan(a) & torch.isnan(b)
    x, y = a.contiguous().view(i), b.contiguous().view(i)
    same = (x == y) | nan | ((a == 0) & (b == 0))
    assert bool(same.all()), "%d of %d values differ" % (int((~same).sum()), same.numel())


INT8_CASES = [
    (1, 1, 1, F32, F32), (15, 7, 2, BF16, F32), (33, 16, 3, F32, BF16), (1000, 64, 1, BF16, F32),
    (4099, 65, 5, BF16, BF16), (2049, 100, 16, F32, F32), (50257, 1000, 5, BF16, F32), (3001, 1024, 17, BF16, F32),
    (4096, 2048, 1, F32, F32), (2000, 8192, 4, BF16, BF16), (777, 8191, 3, F32, F32), (5000, 256, 64, BF16, BF16),
    (3333, 272, 65, BF16, F32), (1031, 512, 130, F32, BF16), (2111, 640, 300, BF16, BF16), (513, 96, 1000, BF16, F32),
    (300, 33, 2100, F32, BF16), (140000, 48, 9, BF16, F32), (6007, 1536, 33, BF16, F32), (257, 2048, 257, BF16, BF16),
    (129, 4096, 48, BF16, F32), (8200, 128, 8, F32, F32),
    (4099, 65, 40, F32, BF16), (3001, 1001, 200, BF16, F32), (1500, 8191, 20, F32, F32), (5000, 1000, 16, BF16, BF16),
    (777, 2040, 16, F32, F32), (9000, 4100, 3, BF16, BF16), (70000, 33, 2, F32, BF16), (3000, 4096, 8, F32, F32),
    (131073, 16, 1, BF16, F32), (500, 8192, 16, BF16, F32),
    # rows of a few bytes: the matrix's last 16 bytes are rows of two tiles
    (2226, 2, 3, BF16, BF16), (2305, 1, 5, F32, F32), (4097, 7, 2, BF16, F32), (70001, 3, 16, F32, BF16), (2066, 15, 4, BF16, F32),
    (9, 2, 3, F32, F32), (16, 1, 2, F32, F32), (17, 1, 2, F32, F32), (2570, 5, 1, F32, F32),
    (700, 2049, 20, BF16, F32), (600, 4097, 16, F32, BF16), (600, 4097, 9, BF16, F32), (900, 2048, 6, F32, F32),
    (900, 2048, 7, F32, F32), (800, 2064, 1, BF16, F32), (1000, 256, 13, BF16, F32),
]


@pytest.mark.parametrize("V,d,B,ht,ot", INT8_CASES)
def test_int8_logits_bitwise(vie, V, d, B, ht, ot):
    say("int8", V, d, B, ht, ot)
    q, scale, h = int8_inputs(V, d, B, ht, V + d + B)
    head = vie.Int8Head(q.cuda(), scale.cuda())
    ref = int8_reference(q, scale, h, ot)
    out = head(h.cuda(), dtype=ot)
    same_bits(out, ref)
    # strided rows that are not 16-byte aligned; nothing between them is written
    view, buf = strided(torch.zeros(B, V, dtype=ot), V + 3, 1)
    head(h.cuda(), out=view)
    same_bits(view, ref)
    assert bool((between(buf, B, V, V + 3, 1) == 77.0).all())


def test_int8_logits_extremes_and_unaligned_rows(vie):
    say("int8 extremes")
    V, d, B = 700, 8192, 3
    q = torch.full((V, d), 127, dtype=torch.int8)
    q[1::2] = -127
    h = torch.ones(B, d)
    scale = torch.ones(V)
    same_bits(vie.Int8Head(q.cuda(), scale.cuda())(h.cuda()), int8_reference(q, scale, h, F32))  # the largest sums
    # tokens with a NaN or an infinity, tiny and huge values, next to an ordinary one
    q, scale, h = int8_inputs(300, 75, 6, F32, 3)
    h[1, 5], h[2, 3], h[3], h[4] = float("nan"), -INF, h[3] * 1e-43, h[4] * 1e37
    dq = torch.zeros(300 * 75 + 5, dtype=torch.int8).cuda()
    view = dq[5:].view(300, 75)  # rows at odd addresses
    view.copy_(q)
    out = vie.Int8Head(view, scale.cuda())(h.cuda())
    same_bits(out, int8_reference(q, scale, h, F32))
    assert bool(torch.isnan(out[1:3]).all()) and not bool(torch.isnan(out[[0, 3, 4, 5]]).any())


@pytest.mark.parametrize("V,d,B", [(600, 64, 3), (301, 272, 14), (500, 2048, 20), (130, 8192, 1), (257, 4096, 6), (900, 1024, 70)])
def test_int8_rows_at_an_odd_address(vie, V, d, B):
    """Rows of a multiple of 16 bytes that begin at an odd address."""
    say("int8 odd address", V, d, B)
    q, scale, h = int8_inputs(V, d, B, BF16, V + d)
    buf = torch.zeros(V * d + 3, dtype=torch.int8).cuda()
    view = buf[3:].view(V, d)
    view.copy_(q)
    same_bits(vie.Int8Head(view, scale.cuda())(h.cuda()), int8_reference(q, scale, h, F32))


def test_int8_head_of_quantized_rows(vie):
    """quantize_rows, Int8Head and the dense head: the int8 logits are the rows' own to the quantization's error."""
    say("int8 of quantize_rows")
    V, d, B = 3000, 256, 9
    W = synth.make_w(V, d, synth.BF16, 5)
    H, _ = synth.make_queries(W, synth.BF16, B, 6)
    Wd, Hd = vie.host_to_torch(W, synth.BF16).cuda(), vie.host_to_torch(H, synth.BF16).cuda()
    q, scale = vie.quantize_rows(Wd, synth.BF16)
    z = vie.Int8Head(q, scale)(Hd)
    same_bits(z, int8_reference(q.cpu(), scale.cpu(), Hd.cpu(), F32))
    exact = Hd.double() @ Wd.double().t()
    # each value is off by half a step on either side: |dz| <= sum |w| xs / 2 + |h| scale / 2 + xs scale / 4
    xs = Hd.double().abs().amax(1) / 127
    bound = (Wd.double().abs().sum(1)[None] * xs[:, None] + Hd.double().abs().sum(1)[:, None] * scale.double()[None]) / 2 \
        + d * xs[:, None] * scale.double()[None] / 4
    assert bool(((z.double() - exact).abs() <= bound * (1 + 1e-5)).all())


# ------------------------------------------------------------------- sampling

def draw_reference(l, ids, u, t, k, p, m):
    """(token, probability, kept) of a row from the definition."""
    at = np.flatnonzero((l > -np.inf) & (ids >= 0))
    if not at.size:
        return -1, 0.0, 0
    at = at[np.lexsort((ids[at], -l[at]))]
    x = l[at].astype(np.float64)
    if not t > 0:
        return int(ids[at[0]]), 1.0, 1
    K = min(k, at.size) if k > 0 else at.size
    with np.errstate(over="ignore", invalid="ignore"):
        w = np.where(x == x[0], 1.0, np.nan_to_num(np.exp((x - x[0]) / np.float64(t))))[:K]
    c = np.cumsum(w)
    n = K
    if p < 1:
        n = min(n, int(np.searchsorted(c, np.float64(p) * c[-1], side="left")) + 1)
    if m > 0:
        n = min(n, int((w >= np.float64(m)).sum()))
    n = max(n, 1)
    j = min(int(np.searchsorted(c[:n], np.float64(u) * c[n - 1], side="right")), n - 1)
    return int(ids[at[j]]), w[j] / c[n - 1], n


def check_draws(got, l, ids, u, t, k, p, m, what):
    tok, prob, kept = (x.cpu().numpy() for x in got)
    B = l.shape[0]
    t, k, p, m = (np.broadcast_to(np.asarray(v), (B,)) for v in (t, k, p, m))  # (numbers in 64 bits, arrays in fp32)
    for b in range(B):
        rt, rp, rk = draw_reference(l[b], ids if ids.ndim == 1 else ids[b], u[b], t[b], k[b], p[b], m[b])
        assert (tok[b], kept[b]) == (rt, rk), "%s row %d: token %d kept %d, expected %d and %d" % (what, b, tok[b], kept[b], rt, rk)
        # fp32 rounding (2^-24) and the integer weights' (2^-45 of the best each, seen against the total)
        assert abs(prob[b] - rp) <= 2.0 ** -23 * rp + 2.0 ** -44, (what, b, prob[b], rp)


SETTINGS = [  # temperature, top_k, top_p, min_p
    (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.1), (0.8, 40, 0.95, 0.02),
    (1.5, 3, 0.5, 0.0), (0.05, 20, 0.99, 0.0), (30.0, 0, 0.9, 0.0), (1.0, 1, 1.0, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 1.0, 1.0),
    (1.0, 0, 0.9999, 0.0), (INF, 0, 0.5, 0.0), (1.0, 0, 1.0, 2.0), (float("nan"), 0, 1.0, 0.0), (1e-6, 0, 0.9, 0.0),
]


def lists(B, k, seed, pad=0, shuffled=False):
    rng = np.random.default_rng(seed)
    lg = -np.sort(-(rng.standard_normal((B, k)) * 2 + 8).astype(np.float32), axis=1)
    ids = np.stack([rng.choice(20 * k + 10, k, replace=False) for _ in range(B)]).astype(np.int32)
    if pad:
        lg[:, k - pad:], ids[:, k - pad:] = -np.inf, -1
    if shuffled:
        for b in range(B):
            o = rng.permutation(k)
            lg[b], ids[b] = lg[b, o], ids[b, o]
    return lg, ids, rng.random(B).astype(np.float32)


def dev(*a):
    return tuple(torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in a)


@pytest.mark.parametrize("B,k,pad,shuffled", [(1, 1, 0, False), (7, 50, 0, False), (5, 64, 13, True), (9, 65, 0, True),
                                              (300, 114, 30, False), (4, 1000, 7, True), (3, 2048, 0, True), (2, 129, 129, False)])
def test_sample_lists(vie, B, k, pad, shuffled):
    lg, ids, u = lists(B, k, B + k, pad, shuffled)
    for t, tk, tp, mp in SETTINGS:
        say("lists", B, k, pad, shuffled, t, tk, tp, mp)
        got = vie.sample(*dev(ids, lg, u), temperature=t, top_k=tk, top_p=tp, min_p=mp)
        check_draws(got, lg, ids, u, t, tk, tp, mp, "lists")


def test_sample_lists_odd_entries(vie):
    """Ties, infinities, NaN, -inf before the end, negative ids, an id twice, u at its ends."""
    say("lists, odd entries")
    n, i = np.float32(np.nan), np.float32(np.inf)
    lg = np.array([[3, 3, 3, 1, 1, -i], [i, i, 5, n, 2, -i], [n, n, n, n, n, n], [-i, 2, -i, 2, 0, n],
                   [7, 6, 6, 5, 5, 4], [0, -0.0, 0, -0.0, -1, -1]], np.float32)
    ids = np.array([[9, 2, 5, 1, 0, 3], [4, 1, 3, 2, 0, 9], [1, 2, 3, 4, 5, 6], [8, 5, 7, 5, -1, 2],
                    [-1, 3, 3, -7, 2, 1], [6, 5, 4, 3, 2, 1]], np.int32)
    for u0 in (0.0, 0.25, 0.5, 0.74, np.float32(1 - 2 ** -24)):
        u = np.full(6, u0, np.float32)
        for t, tk, tp, mp in SETTINGS:
            got = vie.sample(*dev(ids, lg, u), temperature=t, top_k=tk, top_p=tp, min_p=mp)
            check_draws(got, lg, ids, u, t, tk, tp, mp, "odd entries")
    # outside [0, 1): still one of the kept
    for u0 in (1.0, 2.0, np.inf, -1.0, np.nan):
        tok = vie.sample(*dev(ids, lg, np.full(6, u0, np.float32)), top_k=2)[0].cpu().numpy()
        assert tok[0] in (2, 5) and tok[1] in (1, 4) and tok[2] == -1 and tok[3] == 5


def row_logits(B, V, dtype, seed, masked):
    g = torch.Generator().manual_seed(seed)
    z = 1.7 * torch.randn(B, V, generator=g)
    for b in range(B):
        at = torch.randint(0, V, (20,), generator=g)
        z[b, at] += 5
    if masked:
        z[::2][torch.rand(z[::2].shape, generator=g) < 0.9] = -INF
        if B > 1:
            z[-1] = -INF
    u = torch.rand(B, generator=g)
    return z.to(dtype), u


ROW_CASES = [(1, 1, F32, False), (2, 2, BF16, True), (3, 7, BF16, False), (4, 1000, F32, True), (9, 4099, BF16, True),
             (1, 50257, F32, False), (5, 50257, BF16, True), (1, 262144, F32, False), (2, 262147, BF16, False),
             (70, 3001, F32, True), (300, 513, BF16, True), (1100, 129, F32, True), (3, 151936, BF16, True),
             (20, 30011, F32, True), (30, 30011, BF16, False), (140, 20011, F32, False)]


@pytest.mark.parametrize("B,V,dtype,masked", ROW_CASES)
def test_sample_rows(vie, B, V, dtype, masked):
    z, u = row_logits(B, V, dtype, B + V, masked)
    l, ids, un = z.float().numpy(), np.arange(V), u.numpy()
    view, buf = strided(z, V + 5, 3)
    for t, tk, tp, mp in SETTINGS if V < 100000 else SETTINGS[:9]:
        say("rows", B, V, dtype, masked, t, tk, tp, mp)
        got = vie.sample_rows(z.cuda(), u.cuda(), temperature=t, top_k=tk, top_p=tp, min_p=mp)
        check_draws(got, l, ids, un, t, tk, tp, mp, "rows")
        again = vie.sample_rows(view, u.cuda(), temperature=t, top_k=tk, top_p=tp, min_p=mp)
        assert all(torch.equal(x, y) for x, y in zip(got, again))
    assert bool((between(buf, B, V, V + 5, 3) == 77.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sample_rows_settings_per_row(vie, dtype):
    B, V = 64, 9001
    z, u = row_logits(B, V, dtype, 4, True)
    rng = np.random.default_rng(9)
    s = [np.array([SETTINGS[i][c] for i in rng.integers(0, len(SETTINGS), B)], np.float32 if c != 1 else np.int32)
         for c in range(4)]
    t, tk, tp, mp = dev(*s)
    say("rows, settings per row", dtype)
    got = vie.sample_rows(z.cuda(), u.cuda(), temperature=t, top_k=tk, top_p=tp, min_p=mp)
    check_draws(got, z.float().numpy(), np.arange(V), u.numpy(), *s, "per row")
    lg, ids, un = lists(B, 120, 11)
    got = vie.sample(*dev(ids, lg, un), temperature=t, top_k=tk, top_p=tp, min_p=mp)
    check_draws(got, lg, ids, un, *s, "lists per row")


@pytest.mark.parametrize("V", [300, 5000, 70001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sample_rows_ties_and_special_values(vie, V, dtype):
    """Rows of one value, of two, of the lowest, with NaN and infinities, narrow and wide ranges."""
    say("rows, ties", V, dtype)
    g = torch.Generator().manual_seed(V)
    z = torch.zeros(12, V)
    z[1, ::3] = 1.0
    z[2] = LOWEST[dtype]
    z[2, 5] = 0.0
    z[3] = LOWEST[dtype]
    z[4] = torch.randn(V, generator=g)
    z[4, ::2] = float("nan")
    z[5, 7:20] = INF
    z[6] = 20 + 1e-3 * torch.randn(V, generator=g)
    z[7] = 1e30 * torch.randn(V, generator=g)
    z[8] = -torch.arange(V).float()
    z[9] = 10 + torch.randint(0, 3, (V,), generator=g) / 16
    z[10] = 1e-30 * torch.randn(V, generator=g)
    z[11] = torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0)
    z = z.to(dtype)
    u = torch.rand(12, generator=g)
    for t, tk, tp, mp in SETTINGS:
        say("  ", t, tk, tp, mp)
        got = vie.sample_rows(z.cuda(), u.cuda(), temperature=t, top_k=tk, top_p=tp, min_p=mp)
        check_draws(got, z.float().numpy(), np.arange(V), u.numpy(), t, tk, tp, mp, "ties")


@pytest.mark.parametrize("B,V,dtype", [(1, 262144, F32), (3, 151936, BF16), (2, 100003, F32), (70, 40000, BF16)])
@pytest.mark.parametrize("mean,spread", [(20, 2), (0, 0.02), (300, 8)])
def test_sample_rows_rounded_logits(vie, B, V, dtype, mean, spread):
    """Logits of few distinct values (bf16 ones, also held in fp32): thousands of ties at every border."""
    say("rounded", B, V, dtype, mean, spread)
    g = torch.Generator().manual_seed(V + mean)
    z = (mean + spread * torch.randn(B, V, generator=g)).to(BF16).to(dtype)
    z[-1, ::3] = -INF
    u = torch.rand(B, generator=g)
    for t, tk, tp, mp in [(1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (2.0, 9999, 0.95, 0.0), (5.0, 0, 0.99, 0.3), (0.7, 20000, 1.0, 0.0)]:
        say("  ", t, tk, tp, mp)
        got = vie.sample_rows(z.cuda(), u.cuda(), temperature=t, top_k=tk, top_p=tp, min_p=mp)
        check_draws(got, z.float().numpy(), np.arange(V), u.numpy(), t, tk, tp, mp, "rounded")


def test_sample_frequencies(vie):
    """Tokens drawn with evenly spread uniform numbers: each as often as its weight says, to one draw."""
    say("frequencies")
    V, B = 50, 20000
    z = torch.randn(V, generator=torch.Generator().manual_seed(1))
    u = (torch.arange(B) + 0.5) / B
    tok = vie.sample_rows(z.repeat(B, 1).cuda(), u.cuda())[0].cpu()
    freq = torch.bincount(tok.long(), minlength=V).double() / B
    assert bool(((freq - torch.softmax(z.double(), 0)).abs() <= 1.01 / B).all())


# --------------------------------------------------------------- distillation

def distill_reference(s, ids, t, tau, g):
    """Loss [N], gradient [N, V], q and p [N, V] in 64 bits."""
    N, V = s.shape
    tau = np.float64(np.float32(tau))
    x = s.astype(np.float64) / tau
    loss, grad, Q, P = np.zeros(N), np.zeros((N, V)), np.zeros((N, V)), np.zeros((N, V))
    with np.errstate(all="ignore"):
        for n in range(N):
            top = x[n].max()
            e = np.exp(x[n] - top)
            q = e / e.sum()
            logq = x[n] - top - np.log(e.sum())
            ok = (ids[n] >= 0) & (ids[n] < V) & ~(t[n] == -np.inf)
            if not ok.any():
                continue
            y = t[n][ok].astype(np.float64) / tau
            p = np.exp(y - y.max())
            p /= p.sum()
            logp = y - y.max() - np.log(np.exp(y - y.max()).sum())
            at = ids[n][ok]
            terms = np.where(p == 0, 0, p * (logp - logq[at]))
            loss[n] = tau * tau * terms.sum()
            pv = np.zeros(V)
            np.add.at(pv, at, p)
            grad[n] = g[n] * tau * (q - pv)
            Q[n], P[n] = q, pv
    return loss, grad, Q, P


def check_loss(got, ref, tau, V, what):
    # log Z: up to V / 512 + 32 fp32 additions in a row, exponents off by 2^-23 relative (times at most log V + 1
    # on average), all times tau^2; then one rounding
    tol = tau * tau * ((V / 512 + 32) * 2.0 ** -24 + (np.log(V) + 3) * 2.0 ** -22) + 2.0 ** -23 * np.abs(ref)
    with np.errstate(invalid="ignore", over="ignore"):  # (a loss above fp32's range, tau^2 times 1e38, is +inf)
        bad = ~(np.abs(got - ref) <= tol) & ~(np.isnan(got) & np.isnan(ref)) & (got != ref.astype(np.float32))
    assert not bad.any(), (what, got[bad][:4], ref[bad][:4])


def check_grad(got, ref, Q, P, s, tau, g, dtype, what):
    V = s.shape[1]
    with np.errstate(all="ignore"):
        x = np.abs(s.astype(np.float64) - s.max(1, keepdims=True)) / tau
        # q: its exponent is off by 2^-22 relative, its sum as above, a product or two; p: fp32; the type's rounding
        q_tol = Q * ((np.minimum(x, 200) + 4) * 2.0 ** -22 + (V / 512 + 32) * 2.0 ** -24 + (np.log(V) + 3) * 2.0 ** -22)
        tol = np.abs(g)[:, None] * tau * (q_tol + P * 2.0 ** -22) + torch.finfo(dtype).eps / 2 * np.abs(ref) + 1e-37
        bad = ~(np.abs(got - ref) <= tol) & ~(np.isnan(got) & np.isnan(ref)) & (got != ref)  # (tol is NaN beside a NaN)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], ref[bad][:4], np.argwhere(bad)[:4])


def distill_inputs(N, V, k, dtype, seed, kind="plain"):
    rng = np.random.default_rng(seed)
    s = torch.from_numpy((rng.standard_normal((N, V)) * 2).astype(np.float32)).to(dtype)
    t = (rng.standard_normal((N, k)) * 2 + 4).astype(np.float32)
    kk = min(k, V)
    ids = np.full((N, k), -1, np.int32)
    for n in range(N):
        ids[n, :kk] = rng.choice(V, kk, replace=False)
    t[:, kk:] = -np.inf
    if kind == "odd":
        ids[0] = -1                                   # nothing listed
        if N > 1:
            t[1] = -np.inf                            # nothing listed either
        if N > 2 and kk > 2:
            ids[2, 1], ids[2, 2] = V + 5, ids[2, 0]   # out of range, an id twice
        if N > 3:
            s[3, 1:] = LOWEST[dtype]                  # masks of the lowest value
            t[3, 0] = -np.inf
        if N > 4:
            s[4, rng.random(V) < 0.5] = -INF          # masks of -inf, listed ids among them
        if N > 5:
            s[5, V // 2] = float("nan")
        if N > 6:
            s[6] = -INF
        if N > 7:
            t[7, 0] = np.nan
        if N > 8:
            ids[8] = ids[8, 0]                        # one id, k times
        if N > 9:
            s[9, 0] = INF
        if N > 10:
            ids[10] = -1
            s[10] = float("nan")                      # nothing listed over NaN: 0
    return s, ids, t


DISTILL_CASES = [(1, 1, 1, F32, 1.0, "plain"), (2, 2, 3, BF16, 2.0, "plain"), (3, 7, 7, F32, 0.5, "plain"),
                 (13, 1000, 50, BF16, 1.0, "odd"), (13, 1000, 50, F32, 3.0, "odd"), (12, 4099, 2048, F32, 1.0, "odd"),
                 (5, 50257, 64, BF16, 2.0, "plain"), (1, 262144, 50, F32, 1.0, "plain"), (2, 151936, 1000, BF16, 4.0, "odd"),
                 (700, 300, 20, BF16, 1.0, "odd"), (1200, 129, 5, F32, 1.0, "odd"), (40, 9001, 600, F32, 0.05, "odd"),
                 (300, 20000, 64, BF16, 2.0, "odd"),
                 # the step's widths, with and without room to keep a row, one step of it and several
                 (12, 12001, 33, BF16, 1.0, "odd"), (11, 8000, 300, F32, 2.0, "odd"), (11, 30000, 60, BF16, 1.0, "odd"),
                 (11, 30001, 800, BF16, 2.0, "odd"), (11, 31001, 20, F32, 1.0, "odd"), (130, 70001, 40, BF16, 2.0, "odd"),
                 (128, 40003, 1500, F32, 1.0, "odd"), (129, 100003, 300, BF16, 1.0, "odd")]


@pytest.mark.parametrize("N,V,k,dtype,tau,kind", DISTILL_CASES)
def test_distill(vie, N, V, k, dtype, tau, kind):
    say("distill", N, V, k, dtype, tau, kind)
    s, ids, t = distill_inputs(N, V, k, dtype, N + V + k, kind)
    rng = np.random.default_rng(1)
    gl = rng.standard_normal(N).astype(np.float32)
    w = 0.25
    g = gl.astype(np.float64) * w
    sn = s.float().numpy()
    ref, grad, Q, P = distill_reference(sn, ids, t, tau, g)
    sd, (idd, td, gd) = s.cuda(), dev(ids, t, gl)
    loss, stats = vie.distill(sd, idd, td, tau)
    check_loss(loss.cpu().numpy(), ref, tau, V, "loss")
    got = vie.distill_grad(sd, idd, td, stats, tau, gloss=gd, weight=w)
    assert got.dtype == dtype
    check_grad(got.float().cpu().numpy(), grad, Q, P, sn, tau, g, dtype, "grad")
    # both at once, strided, at an odd address: the same bits
    view, buf = strided(s, V + 3, 1)
    out, obuf = strided(torch.zeros(N, V, dtype=dtype), V + 7, 3)
    loss2, got2 = vie.distill_step(view, idd, td, tau, gloss=gd, weight=w, out=out)
    check_loss(loss2.cpu().numpy(), ref, tau, V, "step loss")
    check_grad(got2.float().cpu().numpy(), grad, Q, P, sn, tau, g, dtype, "step grad")
    assert bool((between(buf, N, V, V + 3, 1) == 77.0).all()) and bool((between(obuf, N, V, V + 7, 3) == 77.0).all())
    # in place
    loss3, got3 = vie.distill_step(view, idd, td, tau, gloss=gd, weight=w, out=view)
    assert got3.data_ptr() == view.data_ptr()
    check_loss(loss3.cpu().numpy(), ref, tau, V, "in place loss")
    check_grad(view.float().cpu().numpy(), grad, Q, P, sn, tau, g, dtype, "in place grad")
    same = vie.distill_grad(sd, idd, td, stats, tau, gloss=gd, weight=w, out=sd)
    same_bits(same, got)


def test_distill_gradient_by_differences(vie):
    """Central differences of the 64-bit loss, error h^2 / 6 times a third derivative of at most 1."""
    say("distill differences")
    N, V, k, tau = 3, 40, 6, 2.0
    s, ids, t = distill_inputs(N, V, k, F32, 7)
    one = np.ones(N)
    sn = s.numpy().astype(np.float64)
    h = 1e-3
    diff = np.zeros((N, V))
    for v in range(V):
        up, dn = sn.copy(), sn.copy()
        up[:, v] += h
        dn[:, v] -= h
        diff[:, v] = (distill_reference(up, ids, t, tau, one)[0] - distill_reference(dn, ids, t, tau, one)[0]) / (2 * h)
    loss, grad = vie.distill_step(s.cuda(), *dev(ids, t), tau)
    assert np.abs(grad.cpu().numpy() - diff).max() <= tau * tau * h * h + 1e-5
    check_loss(loss.cpu().numpy(), distill_reference(sn, ids, t, tau, one)[0], tau, V, "loss")


# ------------------------------------------------------------------- together

def test_heads_sampling_and_distillation_together(vie):
    """A decoding step and a training step: lists of the dense head and rows
    of the int8 head give tokens, and the dense head's lists teach the int8
    logits, whose gradient replaces them."""
    say("together")
    V, d, B, k = 5003, 128, 12, 40
    W = synth.make_w(V, d, synth.BF16, 15)
    H, _ = synth.make_queries(W, synth.BF16, B, 16)
    Wd, Hd = vie.host_to_torch(W, synth.BF16).cuda(), vie.host_to_torch(H, synth.BF16).cuda()
    u = torch.rand(B, generator=torch.Generator().manual_seed(2)).cuda()
    ids, lg = vie.DenseHead(Wd, max_batch=B, max_k=k)(Hd, k)
    how = dict(temperature=0.3, top_k=30, top_p=0.9, min_p=0.01)
    got = vie.sample(ids, lg, u, **how)
    # the scattered rows hold the same candidates
    rows = vie.sample_rows(vie.scatter(ids, lg, V), u, **how)
    assert torch.equal(got[0], rows[0]) and torch.equal(got[2], rows[2])
    assert float((got[1] - rows[1]).abs().max()) <= 2.0 ** -23
    check_draws(got, lg.cpu().numpy(), ids.cpu().numpy(), u.cpu().numpy(), 0.3, 30, 0.9, 0.01, "together")
    q, scale = vie.quantize_rows(Wd, synth.BF16)
    z = vie.Int8Head(q, scale)(Hd)
    tok = vie.sample_rows(z, u, **how)
    check_draws(tok, z.cpu().numpy(), np.arange(V), u.cpu().numpy(), 0.3, 30, 0.9, 0.01, "int8 rows")
    zn = z.cpu().numpy()
    ref, grad, Q, P = distill_reference(zn, ids.cpu().numpy(), lg.cpu().numpy(), 1.5, np.full(B, 1 / B))
    loss, g = vie.distill_step(z, ids, lg, 1.5, weight=1 / B, out=z)
    check_loss(loss.cpu().numpy(), ref, 1.5, V, "together")
    check_grad(z.cpu().numpy(), grad, Q, P, zn, 1.5, np.full(B, 1 / B), F32, "together")


@pytest.mark.parametrize("B,V", [(2, 30011), (40, 3001)])
def test_graph_replays_and_side_streams(vie, B, V):
    """Two captured graphs of the chain, replayed in turn with new inputs and
    eager calls between, and a stream of its own."""
    d, k = 96, 20
    say("graphs", B, V)
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randint(-127, 128, (V, d), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    head = vie.Int8Head(q, torch.rand(V, device="cuda", generator=g) * 1e-3)
    ids = torch.argsort(torch.rand(B, V, device="cuda", generator=g), dim=1)[:, :k].to(torch.int32).contiguous()

    def new():
        return (torch.randn(B, d, device="cuda", generator=g), torch.rand(B, device="cuda", generator=g),
                torch.randn(B, k, device="cuda", generator=g))

    def chain(h, u, t):
        z = head(h)
        tok = vie.sample_rows(z, u, temperature=0.9, top_k=0, top_p=0.9)
        lst = vie.sample(ids, t, u, top_p=0.8)
        loss, stats = vie.distill(z, ids, t, 2.0)
        back = vie.distill_grad(z, ids, t, stats, 2.0)
        loss2, grad = vie.distill_step(z, ids, t, 2.0, out=z)
        return (*tok, *lst, loss, back, loss2, grad)

    graphs = []
    for _ in range(2):
        held = new()
        chain(*held)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = chain(*held)
        graphs.append((gr, held, out))
    for rep in range(3):
        for gr, held, out in graphs:
            for x, y in zip(held, new()):
                x.copy_(y)
            want = [x.clone() for x in chain(*held)]
            gr.replay()
            torch.cuda.synchronize()
            for x, y in zip(out, want):
                assert torch.equal(x, y), rep
    args = new()
    want = chain(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = chain(*args)
    side.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_top_p_next_to_one(vie):
    """The sums' integers have more bits than fp64: a product with top_p < 1 may round past the sum itself."""
    say("top_p next to one")
    p = float(np.nextafter(1.0, 0.0))
    for B, V, dtype in ((64, 9000, F32), (64, 9000, BF16), (3, 300000, F32)):
        z, u = row_logits(B, V, dtype, V, False)
        zd, ud = z.cuda(), u.cuda()
        near, one = vie.sample_rows(zd, ud, top_p=p), vie.sample_rows(zd, ud, top_p=1.0)
        assert torch.equal(near[0], one[0]) and torch.equal(near[1], one[1])
        assert bool((near[2] >= V // 2).all()) and bool((near[2] <= one[2]).all())
    lg = torch.randn(500, 100, generator=torch.Generator().manual_seed(4)).sort(dim=1, descending=True)[0].contiguous()
    ids = torch.arange(100, dtype=torch.int32).repeat(500, 1).contiguous()
    u = torch.rand(500, generator=torch.Generator().manual_seed(5))
    near, one = (vie.sample(ids.cuda(), lg.cuda(), u.cuda(), top_p=x) for x in (p, 1.0))
    assert torch.equal(near[0], one[0]) and torch.equal(near[2], one[2])


def test_top_k_beyond_32_bits_is_no_limit(vie):
    say("large top_k")
    z, u = row_logits(3, 5000, F32, 8, False)
    for big, plain in (((1 << 40) + 1, 0), (-(1 << 40) + 1, 0), ((1 << 31) - 1, 0)):
        for x, y in zip(vie.sample_rows(z.cuda(), u.cuda(), top_k=big, top_p=0.9),
                        vie.sample_rows(z.cuda(), u.cuda(), top_k=plain, top_p=0.9)):
            assert torch.equal(x, y)


def test_results_do_not_change_between_runs(vie):
    say("run to run")
    z, u = row_logits(6, 40009, BF16, 8, True)
    zd, ud = z.cuda(), u.cuda()
    s, ids, t = distill_inputs(20, 30000, 70, BF16, 5)
    sd, (idd, td) = s.cuda(), dev(ids, t)
    first = None
    for _ in range(4):
        got = [*vie.sample_rows(zd, ud, top_p=0.97), *vie.distill_step(sd, idd, td, 2.0)]
        torch.cuda.synchronize()
        if first is None:
            first = got
        assert all(torch.equal(x, y) for x, y in zip(got, first))


def test_streams_at_once(vie):
    """Calls on two streams that run at the same time do not meet in a workspace."""
    say("two streams")
    work = []
    for k in range(2):
        z, u = row_logits(4, 60000, F32, 20 + k, False)
        q, scale, h = int8_inputs(20000, 200, 70, BF16, 30 + k)
        s, ids, t = distill_inputs(6, 150000, 30, BF16, 40 + k)
        work.append([x.cuda() for x in (z, u, q, scale, h, s, *(torch.from_numpy(np.ascontiguousarray(y)) for y in (ids, t)))])

    def calls(z, u, q, scale, h, s, ids, t):
        return [*vie.sample_rows(z, u, top_p=0.9), vie.Int8Head(q, scale)(h), *vie.distill_step(s, ids, t, 2.0)]

    want = [calls(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for st, w in zip(streams, work):
            with torch.cuda.stream(st):
                got.append(calls(*w))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_offsets_past_32_bits(vie):
    """Rows 2.4 GB apart, and int8 rows of 2.5 GB in all."""
    V, R, ld = 5003, 3, 1_200_000_000
    say("offsets: rows", V, R, ld)
    buf = torch.empty(ld * (R - 1) + V, dtype=BF16, device="cuda")
    far = buf.as_strided((R, V), (ld, 1))
    z, u = row_logits(R, V, BF16, 3, False)
    far.copy_(z)
    got = vie.sample_rows(far, u.cuda(), top_p=0.9)
    assert all(torch.equal(x, y) for x, y in zip(got, vie.sample_rows(z.cuda(), u.cuda(), top_p=0.9)))
    s, ids, t = distill_inputs(R, V, 20, BF16, 4)
    idd, td = dev(ids, t)
    want = vie.distill_step(s.cuda(), idd, td, 2.0)
    far.copy_(s)
    loss, grad = vie.distill_step(far, idd, td, 2.0, out=far)
    assert torch.equal(loss, want[0]) and torch.equal(grad, want[1])
    q, scale, h = int8_inputs(V, 96, R, BF16, 5)
    vie.Int8Head(q.cuda(), scale.cuda())(h.cuda(), out=far)
    same_bits(far, int8_reference(q, scale, h, BF16))
    del buf, far, grad
    V, d = 300007, 8192
    say("offsets: int8 rows", V, d)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randint(-127, 128, (V, d), dtype=torch.int8, device="cuda", generator=g)
    scale = torch.rand(V, device="cuda", generator=g) * 1e-3
    for B in (2, 70):
        h = torch.randn(B, d, generator=torch.Generator().manual_seed(B))
        out = vie.Int8Head(q, scale)(h.cuda())
        for part in (slice(0, 700), slice(262100, 262200), slice(V - 700, V)):
            same_bits(out[:, part].contiguous(), int8_reference(q[part].cpu(), scale[part].cpu(), h, F32))


def test_many_short_rows(vie):
    """More rows than a launch dimension takes at once."""
    N, V, k = 40000, 17, 3
    say("many rows", N, V)
    s, ids, t = distill_inputs(N, V, k, F32, 9)
    idd, td = dev(ids, t)
    ref, grad, Q, P = distill_reference(s.numpy(), ids, t, 1.0, np.ones(N))
    loss, stats = vie.distill(s.cuda(), idd, td, 1.0)
    back = vie.distill_grad(s.cuda(), idd, td, stats, 1.0)
    loss2, grad2 = vie.distill_step(s.cuda(), idd, td, 1.0)
    for x, y in ((loss, back), (loss2, grad2)):
        check_loss(x.cpu().numpy(), ref, 1.0, V, "many rows")
        check_grad(y.cpu().numpy(), grad, Q, P, s.numpy(), 1.0, np.ones(N), F32, "many rows")
    z, u = row_logits(3000, 40, F32, 1, False)
    got = vie.sample_rows(z.cuda(), u.cuda(), top_k=7, top_p=0.8)
    check_draws(got, z.numpy(), np.arange(40), u.numpy(), 1.0, 7, 0.8, 0.0, "many rows")
    lg, li, un = lists(20000, 9, 2)
    check_draws(vie.sample(*dev(li, lg, un), top_p=0.7), lg, li, un, 1.0, 0, 0.7, 0.0, "many lists")


def leaf(t):
    return t.detach().clone().requires_grad_()


@pytest.mark.parametrize("N,V,k,dtype,tau,kind", [(1, 1, 1, F32, 1.0, "plain"), (13, 1000, 50, BF16, 1.0, "odd"),
                                                  (12, 4099, 2048, F32, 3.0, "odd"), (300, 20000, 64, BF16, 2.0, "odd")])
def test_distill_is_recorded_by_autograd(vie, N, V, k, dtype, tau, kind):
    """A backward pass through distill gives distill_grad's values, whatever else is in the loss."""
    say("autograd", N, V, k, dtype, tau, kind)
    s, ids, t = distill_inputs(N, V, k, dtype, N + V, kind)
    idd, td = dev(ids, t)
    w = torch.randn(N, generator=torch.Generator().manual_seed(1)).cuda()
    z = leaf(s.cuda())
    loss, stats = vie.distill(z, idd, td, tau)
    plain, plain_stats = vie.distill(z.detach(), idd, td, tau)
    assert loss.requires_grad and not stats.requires_grad and not plain.requires_grad
    same_bits(loss.detach(), plain)
    same_bits(stats, plain_stats)
    for total, gloss in (((loss * w).sum(), w), (loss.sum(), None), (loss.mean(), torch.full_like(w, 1 / N))):
        (got,) = torch.autograd.grad(total, z, retain_graph=True)
        same_bits(got, vie.distill_grad(z.detach(), idd, td, stats, tau, gloss=gloss))
    with torch.no_grad():
        assert not vie.distill(z, idd, td, tau)[0].requires_grad
    # beside another term, through a layer before, in strided rows
    h = torch.randn(N, 8, generator=torch.Generator().manual_seed(2)).cuda()
    W = leaf(torch.randn(V, 8, generator=torch.Generator().manual_seed(3)).cuda())

    def logits():
        y = (h @ W.t()).to(dtype)
        return torch.cat([y, y[:, :1]], 1)[:, :V]

    y = logits()
    (0.5 * y.float().square().sum() + vie.distill(y, idd, td, tau)[0].sum()).backward()
    yd = y.detach()
    dy = vie.distill_grad(yd, idd, td, vie.distill(yd, idd, td, tau)[1], tau)
    y2 = logits()
    (want,) = torch.autograd.grad(y2, W, (yd.float() + dy.float()).to(dtype))
    # (two terms of y's type are added in another order: a rounding of each and of their sum, through 8 products)
    ok = torch.isfinite(want)
    size = (yd.float().abs() + dy.float().abs()).nan_to_num(0, 0, 0).t() @ h.abs()
    tol = 4 * torch.finfo(dtype).eps * size + 1e-5
    assert bool(((W.grad - want).abs() <= tol)[ok].all()) and bool((ok == torch.isfinite(W.grad)).all())


def test_distill_step_gives_its_gradient_once(vie):
    """The step's gradient is its second result; a backward pass from its loss says so instead of giving nothing."""
    say("autograd, step")
    s, ids, t = distill_inputs(5, 300, 20, F32, 3)
    idd, td = dev(ids, t)
    z = leaf(s.cuda())
    loss, grad = vie.distill_step(z, idd, td, 2.0, weight=0.2)
    assert not grad.requires_grad
    z.backward(grad)
    same_bits(z.grad, vie.distill_step(z.detach(), idd, td, 2.0, weight=0.2)[1])
    with pytest.raises(RuntimeError, match="second result"):
        (z.square().mean() + loss.mean()).backward()
    assert not vie.distill_step(z.detach(), idd, td, 2.0)[0].requires_grad
    with torch.no_grad():
        assert not vie.distill_step(z, idd, td, 2.0)[0].requires_grad
    with pytest.raises(ValueError, match="detach"):
        vie.distill(z, idd, leaf(td), 2.0)


def test_autograd_sees_tensors_written_over(vie):
    """A tensor that a backward pass needs is not overwritten behind its back."""
    say("autograd, out=")
    V, d, B, k = 500, 64, 4, 10
    q, scale, h = int8_inputs(V, d, B, F32, 1)
    head = vie.Int8Head(q.cuda(), scale.cuda())
    s, ids, t = distill_inputs(B, V, k, F32, 2)
    idd, td = dev(ids, t)
    stats = vie.distill(s.cuda(), idd, td)[1]
    for write in (lambda y: head(h.cuda(), out=y), lambda y: vie.distill_step(y.detach(), idd, td, out=y),
                  lambda y: vie.distill_grad(y.detach(), idd, td, stats, out=y)):
        y = leaf(s.cuda()).exp()  # (whose backward pass needs y itself)
        write(y)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
        z = leaf(s.cuda()) * 1.0
        loss = vie.distill(z, idd, td)[0]
        write(z)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.sum().backward()


def test_recorded_distillation_in_a_graph(vie):
    """Forward and backward passes captured, replayed with new inputs, with eager passes between."""
    say("autograd, captured")
    N, V, k = 6, 3001, 12
    s, ids, t = distill_inputs(N, V, k, BF16, 11)
    idd, td = dev(ids, t)
    w = torch.rand(N, generator=torch.Generator().manual_seed(4)).cuda()

    def both(z):
        loss = vie.distill(z, idd, td, 2.0)[0]
        return loss.detach(), torch.autograd.grad((loss * w).sum(), z)[0]

    both(leaf(s.cuda()))
    torch.cuda.synchronize()
    z = leaf(s.cuda())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(z)
    for rep in range(3):
        with torch.no_grad():
            z.copy_(torch.randn(N, V, generator=torch.Generator().manual_seed(rep)))
        want = both(leaf(z))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(out, want):
            same_bits(x, y)


@pytest.mark.parametrize("N,V,dtype", [(12, 4099, F32), (40, 9001, F32), (130, 20001, BF16), (130, 70001, F32), (3, 150001, F32)])
def test_distill_step_uses_one_sum_a_row(vie, N, V, dtype):
    """Equal logits of a row have equal gradients, to the bit, whichever thread
    stores them; and strides and places change no bit of a step."""
    say("one sum a row", N, V, dtype)
    s, ids, t = distill_inputs(N, V, 9, dtype, N + V)
    s[:, ::2] = 1.25
    idd, td = dev(ids, t)
    loss, grad = vie.distill_step(s.cuda(), idd, td, 2.0)
    same = grad[:, ::2].cpu().float()
    listed = torch.zeros(N, V, dtype=torch.bool).scatter_(1, torch.from_numpy(ids).long(), True)[:, ::2]
    for n in range(N):
        values = same[n][~listed[n]].unique()
        assert values.numel() == 1, (n, values)
    view, _ = strided(s, V + 3, 1)
    out, _ = strided(torch.zeros(N, V, dtype=dtype), V + 7, 3)
    for x in (vie.distill_step(view, idd, td, 2.0, out=out), vie.distill_step(view, idd, td, 2.0, out=view)):
        same_bits(x[0], loss)
        same_bits(x[1], grad)


def test_distill_sums_of_very_long_rows(vie):
    """Equal logits below a thread's largest round the same way in every
    addition, so that a long fp32 sum runs away from the true one (by 4e-4
    after 32768 of these, 2e-4 after 16384)."""
    V, x, tops = 1 << 24, 3.5, 2048
    Z = tops + (V - tops) * np.exp(-x)
    # fp32 sums of 512 terms and the merges after them, the exponents; the loss is log Z
    tol = (512 + 32) * 2.0 ** -24 + (np.log(V) + 3) * 2.0 ** -22 + 2.0 ** -23 * np.log(Z)
    for N, dtype in ((257, BF16), (130, F32)):
        say("long rows", N, V, dtype)
        s = torch.full((N, V), -x, dtype=dtype, device="cuda")
        s[:, :4 * tops:4] = 0.0
        ids = torch.full((N, 1), 8, dtype=torch.int32, device="cuda")
        t = torch.zeros(N, 1, device="cuda")
        loss, stats = vie.distill(s, ids, t)
        assert float((loss.double() - np.log(Z)).abs().max()) <= tol
        assert float((stats[:, 1].double() / Z - 1).abs().max()) <= tol
        s, ids, t = s[:130], ids[:130], t[:130]  # (in one kernel)
        loss, grad = vie.distill_step(s, ids, t, out=s)
        assert float((loss.double() - np.log(Z)).abs().max()) <= tol
        half = torch.finfo(dtype).eps / 2
        for at, want in ((slice(4 * tops, V), np.exp(-x) / Z), (slice(0, 8, 4), 1 / Z), (slice(8, 9), 1 / Z - 1)):
            worst = max(float((grad[n, at].double() / want - 1).abs().max()) for n in range(0, 130, 9))
            assert worst <= tol + 2.0 ** -21 + half, (at, worst)
        del s, grad


@pytest.mark.parametrize("dtype,V", [(BF16, 300007), (F32, 270001), (BF16, 620001)])
def test_distill_odd_values_in_long_rows(vie, dtype, V):
    """Rows of more than 512 terms a thread, among them masked ones and ones with NaN and infinities."""
    say("long odd rows", dtype, V)
    n, copies, k, tau, w = 12, 22, 30, 2.0, 0.5
    s, ids, t = distill_inputs(n, V, k, dtype, V, "odd")
    g = np.full(n, w)
    sn = s.float().numpy()
    ref, grad, Q, P = distill_reference(sn, ids, t, tau, g)
    sd, idd, td = s.cuda().repeat(copies, 1), *(x.repeat(copies, 1) for x in dev(ids, t))
    loss, stats = vie.distill(sd, idd, td, tau)
    back = vie.distill_grad(sd, idd, td, stats, tau, weight=w)
    step_loss, step_grad = vie.distill_step(sd, idd, td, tau, weight=w, out=sd)
    for l, d, what in ((loss, back, "apart"), (step_loss, step_grad, "step")):
        check_loss(l[:n].cpu().numpy(), ref, tau, V, what)
        check_grad(d[:n].float().cpu().numpy(), grad, Q, P, sn, tau, g, dtype, what)
        for c in range(1, copies):
            same_bits(l[c * n:c * n + n], l[:n])
            i = torch.int32 if dtype == F32 else torch.int16
            assert torch.equal(d[c * n:c * n + n].view(i), d[:n].view(i))


@pytest.mark.parametrize("V,d,B", [((1 << 26) + 77, 17, 33), ((1 << 30) + 70, 1, 17)])
def test_int8_more_rows_than_a_launch_has_threads(vie, V, d, B):
    say("int8, many rows", V, d, B)
    g = torch.Generator(device="cuda").manual_seed(V)
    q = torch.randint(-127, 128, (V, d), dtype=torch.int8, device="cuda", generator=g)
    scale = torch.rand(V, device="cuda", generator=g)
    h = torch.randn(B, d, generator=torch.Generator().manual_seed(B))
    out = vie.Int8Head(q, scale)(h.cuda(), dtype=BF16)
    for at in (0, (1 << 24) - 50, (1 << 26) - 50, (1 << 28) - 50, (1 << 30) - 50, V - 100):
        part = slice(at, at + 100)
        if at < V:
            same_bits(out[:, part].contiguous(), int8_reference(q[part].cpu(), scale[part].cpu(), h, BF16))


def test_quantize_more_rows_than_a_launch_has_threads(vie):
    V, d = (1 << 26) + 77, 3
    say("quantize_rows, many rows", V, d)
    W = torch.randn(V, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    q, scale = vie.quantize_rows(W, synth.F32)
    for at in (0, 300, 1 << 24, (1 << 26) - 50, V - 100):
        w = W[at:at + 100].cpu().numpy()
        sc = (np.abs(w).max(1) / np.float32(127)).astype(np.float32)
        assert np.array_equal(scale[at:at + 100].cpu().numpy(), sc)
        assert np.array_equal(q[at:at + 100].cpu().numpy(), np.clip(np.rint((w / sc[:, None]).astype(np.float32)), -127, 127))


def test_the_largest_vocabulary(vie):
    """2^31 - 1 ids, the most that the calls accept."""
    V = (1 << 31) - 1
    say("largest vocabulary")
    s = torch.full((1, V), -20.0, dtype=BF16, device="cuda")
    tops = [5, 1 << 30, V - 1]
    s[0, tops] = torch.tensor([1.0, 3.0, 2.0], dtype=BF16, device="cuda")
    w = np.exp(np.array([3.0, 2.0, 1.0]) - 3)
    order = [1 << 30, V - 1, 5]
    for u, at in ((0.0, 0), (0.66, 0), (0.67, 1), (0.9, 1), (0.92, 2), (0.999, 2)):
        tok, prob, kept = vie.sample_rows(s, torch.full((1,), u, device="cuda"), top_k=3)
        assert (int(tok), int(kept)) == (order[at], 3) and abs(float(prob) - w[at] / w.sum()) <= 2.0 ** -23
    tok, prob, kept = vie.sample_rows(s, torch.zeros(1, device="cuda"), temperature=0.0)
    assert (int(tok), float(prob), int(kept)) == (1 << 30, 1.0, 1)
    s.fill_(1.0)  # all alike: the token follows from its number
    tok, prob, kept = vie.sample_rows(s, torch.full((1,), 0.75, device="cuda"))
    assert (int(tok), int(kept)) == (int(0.75 * V), V) and abs(float(prob) * V - 1) <= 2.0 ** -23
    s.fill_(-20.0)
    s[0, tops] = torch.tensor([1.0, 3.0, 2.0], dtype=BF16, device="cuda")
    ids = torch.tensor([tops + [-1, 77]], dtype=torch.int32, device="cuda")
    t = torch.tensor([[0.0, 1.0, 2.0, 9.0, -1.0]], device="cuda")
    Z = w.sum() + (V - 3) * np.exp(-23.0)
    logq = np.array([-2.0, 0.0, -1.0, -23.0]) - np.log(Z)
    y = np.array([0.0, 1.0, 2.0, -1.0])
    p = np.exp(y) / np.exp(y).sum()
    want = float((p * (np.log(p) - logq)).sum())
    loss, grad = vie.distill_step(s, ids, t, out=s)
    assert abs(float(loss) - want) <= (512 + 32) * 2.0 ** -24 + (np.log(V) + 3) * 2.0 ** -22 + 2.0 ** -23 * want
    for at, pj, lq in zip(tops + [77, 100, V - 2], list(p) + [0, 0], list(logq) + [logq[3]] * 2):
        q = np.exp(lq)
        assert abs(float(grad[0, at]) - (q - pj)) <= 2.0 ** -8 * abs(q - pj) + 1e-4 * q + 2.0 ** -22 * pj
    del s, grad
    q = torch.randint(-127, 128, (V, 1), dtype=torch.int8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    scale = torch.ones(V, device="cuda")
    scale[-200:] = 0.25
    h = torch.tensor([[3.5]])
    out = vie.Int8Head(q, scale)(h.cuda(), dtype=BF16)
    for at in (0, (1 << 30) - 50, V - 250):
        part = slice(at, at + 250)
        same_bits(out[:, part].contiguous(), int8_reference(q[part].cpu(), scale[part].cpu(), h, BF16))


@pytest.mark.parametrize("V,d,B", [(50257, 1000, 32), (3001, 65, 17), (2049, 1001, 31), (70001, 3, 20), (333, 2047, 18),
                                   (17, 1, 17), (65, 63, 32), (1000, 2033, 29), (64, 2041, 24), (1, 2000, 25)])
@pytest.mark.parametrize("ht,ot,odd", [(F32, BF16, 0), (BF16, F32, 0), (BF16, BF16, 1), (F32, F32, 7)])
def test_int8_unaligned_rows_read_for_every_16_tokens(vie, V, d, B, ht, ot, odd):
    """17 to 32 tokens over rows of up to 2048 bytes that are no multiple of
    16: pieces that reach into the next row, and past the matrix's end."""
    say("int8 17-32 tokens, unaligned", V, d, B, ht, ot, odd)
    q, scale, h = int8_inputs(V, d, B, ht, V + d)
    buf = torch.full((odd + V * d,), 127, dtype=torch.int8).cuda()
    view = buf[odd:].view(V, d)
    view.copy_(q)
    head, ref = vie.Int8Head(view, scale.cuda()), int8_reference(q, scale, h, ot)
    same_bits(head(h.cuda(), dtype=ot), ref)
    out, obuf = strided(torch.zeros(B, V, dtype=ot), V + 3, 1)
    head(h.cuda(), out=out)
    same_bits(out, ref)
    assert bool((between(obuf, B, V, V + 3, 1) == 77.0).all())


@pytest.mark.parametrize("V,d,B", [(300, 48, 17), (1001, 2064, 40), (77, 8192, 33), (2000, 112, 300)])
def test_int8_rows_at_an_odd_address_and_many_tokens(vie, V, d, B):
    say("int8 odd address, many tokens", V, d, B)
    q, scale, h = int8_inputs(V, d, B, F32, V + d)
    buf = torch.full((9 + V * d,), 127, dtype=torch.int8).cuda()
    view = buf[9:].view(V, d)
    view.copy_(q)
    same_bits(vie.Int8Head(view, scale.cuda())(h.cuda()), int8_reference(q, scale, h, F32))


@pytest.mark.parametrize("V,dtype", [(40, F32), (17500, BF16), (30000, F32), (81000, F32), (90000, BF16)])
def test_sample_rows_stays_in_its_workspace(vie, V, dtype):
    """A workspace for the most rows serves fewer; nothing is written past the
    size asked for, with rows that are drawn from bins, ties and digits."""
    say("sampling workspace", V, dtype)
    most = 200
    need = vie._workspace_bytes("vie_sample_rows_workspace", V, most)
    ws = torch.empty(need + 4096, dtype=torch.uint8, device="cuda")
    z, u = row_logits(most, V, dtype, V, False)
    z[::3] = 2.5                                                                         # ties
    z[1::3] = 10 + 1e-2 * torch.randn(z[1::3].shape, generator=torch.Generator().manual_seed(1)).to(dtype)  # one bin, many values
    z, u = z.cuda(), u.cuda()
    prm = vie.SamplingParams(1.0, 0.9, 0.0, 0)
    for B in (1, 2, 7, 8, 9, 31, 127, 128, 129, most):
        own = vie._workspace_bytes("vie_sample_rows_workspace", V, B)
        assert own <= need
        want = vie.sample_rows(z[:B], u[:B], top_p=0.9)
        got = vie._drawn(B, z.device)
        ws.fill_(0x5A)
        vie._check(vie.lib.vie_sample_rows(z.data_ptr(), vie._dtype_of_tensor(z), V, V, B, vie.C.byref(prm), u.data_ptr(),
                                           *(x.data_ptr() for x in got), ws.data_ptr(), need, vie._raw_stream(z.device)))
        assert all(torch.equal(x, y) for x, y in zip(got, want)), B
        assert bool((ws[own:] == 0x5A).all()), B


def test_the_most_rows(vie):
    """65535 rows, the most that the calls accept."""
    B = 65535
    say("most rows")
    z, u = row_logits(B, 21, BF16, 5, False)
    got = vie.sample_rows(z.cuda(), u.cuda(), top_k=5, top_p=0.8)
    some = np.r_[0:300, 32700:33000, B - 300:B]
    check_draws([x[some] for x in got], z.float().numpy()[some], np.arange(21), u.numpy()[some], 1.0, 5, 0.8, 0.0, "most rows")
    lg, ids, un = lists(B, 3, 6)
    got = vie.sample(*dev(ids, lg, un), top_p=0.9)
    check_draws([x[some] for x in got], lg[some], ids[some], un[some], 1.0, 0, 0.9, 0.0, "most lists")
    s, ids, t = distill_inputs(B, 9, 3, BF16, 7)
    idd, td = dev(ids, t)
    sn = s.float().numpy()[some]
    ref, grad, Q, P = distill_reference(sn, ids[some], t[some], 2.0, np.ones(some.size))
    loss, stats = vie.distill(s.cuda(), idd, td, 2.0)
    back = vie.distill_grad(s.cuda(), idd, td, stats, 2.0)
    for l, g in ((loss, back), vie.distill_step(s.cuda(), idd, td, 2.0)):
        check_loss(l.cpu().numpy()[some], ref, 2.0, 9, "most rows")
        check_grad(g.float().cpu().numpy()[some], grad, Q, P, sn, 2.0, np.ones(some.size), BF16, "most rows")
    for d in (16, 23):
        q, scale, h = int8_inputs(40, d, B, BF16, d)
        same_bits(vie.Int8Head(q.cuda(), scale.cuda())(h.cuda()), int8_reference(q, scale, h, F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_arguments_between_the_rows_of_others(vie, dtype):
    """Logits and their gradient in the two halves of wider rows, and small arrays behind a row."""
    say("between rows", dtype)
    N, V, k = 6, 1001, 8
    s, ids, t = distill_inputs(N, V, k, dtype, 3)
    idd, td = dev(ids, t)
    u = torch.rand(N, generator=torch.Generator().manual_seed(1)).cuda()
    want = [*vie.distill_step(s.cuda(), idd, td, 2.0), *vie.sample_rows(s.cuda(), u, top_p=0.9)]
    wide = torch.full((N, 2 * V + 30), 77.0, dtype=dtype, device="cuda")
    z, g = wide[:, :V], wide[:, V:2 * V]
    z.copy_(s)
    stats = vie.distill(z, idd, td, 2.0)[1]
    vie.distill_grad(z, idd, td, stats, 2.0, out=g)
    back = g.clone()
    got = [*vie.distill_step(z, idd, td, 2.0, out=g), *vie.sample_rows(z, u, top_p=0.9)]
    for x, y in zip(got, want):
        same_bits(x, y) if x.is_floating_point() else None
        assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float()))
    same_bits(back, vie.distill_grad(s.cuda(), idd, td, stats, 2.0))
    same_bits(z, s)
    assert bool((wide[:, 2 * V:] == 77.0).all())
    q, scale, h = int8_inputs(V, 33, N, F32, 4)
    vie.Int8Head(q.cuda(), scale.cuda())(h.cuda(), out=g)
    same_bits(g, int8_reference(q, scale, h, dtype))
    same_bits(z, s)
    # the token's array in the gap behind row 2
    ld = 2048
    buf = torch.zeros(N * ld, dtype=dtype, device="cuda")
    rows = buf.view(N, ld)[:, :V]
    rows.copy_(s)
    gap = buf[2 * ld + 1024:].view(torch.int32)[:N]
    prm = vie.SamplingParams(1.0, 0.9, 0.0, 0)
    n = vie._workspace_bytes("vie_sample_rows_workspace", V, N)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    vie._check(vie.lib.vie_sample_rows(rows.data_ptr(), vie._dtype_of_tensor(rows), V, ld, N, vie.C.byref(prm), u.data_ptr(),
                                       gap.data_ptr(), None, None, ws.data_ptr(), n, vie._raw_stream(rows.device)))
    assert torch.equal(gap, want[2])
    same_bits(rows, s)
