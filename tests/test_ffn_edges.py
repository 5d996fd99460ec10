"""The operators of a layer's feed-forward half where few bits are left, numbers are tiny or far apart, and kernels run that ordinary
sizes do not reach.  Bounds as in test_ffn_ops.py, and where a test says so, of one rounding alone."""
import numpy as np
import pytest

from oracle import ffn_oracle as want
from test_ffn_ops import CUT, U, Bank, choices, experts_check, f64, mixing, near, norm_case, normal

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def w2():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_06753_amd import binding
    return binding


class MadeBank(Bank):
    """Experts of codes [E, K, N] and scales [E, K/G, N] that a test makes itself."""

    def __init__(self, w2, hidden, inter, G, up, down):
        self.hidden, self.inter, self.E, self.G, self.zero = hidden, inter, len(up[0]), G, 2
        self.parts, blobs = [], []
        for codes, scales in (up, down):
            scales = torch.tensor(np.asarray(scales), dtype=torch.float32).bfloat16()
            codes = np.asarray(codes, dtype=np.uint8)
            blobs.append(torch.stack([w2.prepack(torch.from_numpy(c).cuda(), s.cuda(), G) for c, s in zip(codes, scales)]))
            self.parts.append((codes, scales.double().numpy()))
        self.experts = w2.Experts(*blobs, hidden=hidden, inter=inter, G=G)


# ------------------------------------------------------------------ experts: what a row's sums keep
@pytest.mark.gpu
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("M,E", [(5, 2), (40, 64), (40, 2), (300, 2)])        # in two launches, few rows an expert, many
def test_experts_that_all_but_cancel(w2, M, E, G):
    """Two experts whose results differ by 2^-7 of themselves, one less the other: what is left has the usual relative error only if
    either sum is kept in 32 bits until they meet.  Their h and their products are the same bits, so that the errors of h and of the products
    shrink with the difference; the sums' roundings do not: at most 16 of 2^-24 of the magnitude for each of two, 2^-19 together."""
    hidden, inter = 512, 256
    rng = np.random.default_rng(M + E + G)
    up = rng.integers(0, 4, (1, hidden, 2 * inter)).repeat(E, 0), rng.uniform(0.005, 0.05, (1, hidden // G, 2 * inter)).repeat(E, 0)
    scale = np.full((E, inter // G, hidden), 2.0 ** -5)
    scale[1] *= 1.0 + 2.0 ** -7                               # eight bits
    bank = MadeBank(w2, hidden, inter, G, up, (rng.integers(0, 4, (1, inter, hidden)).repeat(E, 0), scale))
    x = normal(M, M, hidden)
    ids = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda").repeat(M, 1)
    weights = torch.tensor([[1.0, -1.0]], device="cuda").repeat(M, 1)
    ref, mag, h_err = want.experts(f64(x), ids.cpu().numpy(), f64(weights), bank.weights(0), bank.weights(1))
    y = w2.moe_experts(bank.experts, x, ids, weights)
    near(y, ref, U * np.abs(ref) + 2.0 ** -8 * ((U + CUT) * mag + CUT * h_err) + 2.0 ** -19 * mag, "two experts that all but cancel")
    off, norm = np.linalg.norm(f64(y) - ref), np.linalg.norm(ref)
    assert off <= 0.0036 * norm + 2.0 ** -19 * np.linalg.norm(mag), f"{off / norm:.4f} off"


# ------------------------------------------------------------------ experts: up to 64 choices, local memory around 64 KiB
@pytest.mark.gpu
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("hidden,top", [(3584, 7), (3584, 8), (4096, 6), (4096, 7), (4096, 8), (5120, 5), (5120, 6), (7168, 4)])
def test_experts_rows_around_64_kib(w2, hidden, top, G):
    """One token and two: rows that fill 52 to 66 KiB of local memory, and 12 KiB beside them."""
    bank = Bank(w2, hidden, 256, top + 1, G, seed=hidden + top)
    for M in (1, 2):
        experts_check(w2, bank, normal(M, M, hidden), choices(M, top + 1, top, M), mixing(M, top, M), what=f"hidden={hidden} top={top} M={M}")


# ------------------------------------------------------------------ the router where probabilities run out of 64 bits
def renormalised(l, ids, scale):
    """scale * exp(l - largest) / sum over the chosen ones: what p / (sum of p) is wherever every p is proportional to exp(l)."""
    c = np.take_along_axis(l, ids, 1)
    w = np.exp(c - c.max(1, keepdims=True))
    return scale * w / w.sum(1, keepdims=True)


@pytest.mark.gpu
@pytest.mark.parametrize("E,top,groups", [(40, 5, 1), (128, 8, 1), (256, 8, 8), (1000, 64, 4)])
@pytest.mark.parametrize("low", [-650.0, -720.0, -2000.0])
def test_route_sigmoids_of_nothing_are_renormalised(w2, E, top, groups, low):
    """Scores around -650 to -2000, where a sigmoid is exp(l) and below what 64 bits hold: the weights are their finite quotients."""
    M, K = 9, 512
    x, W = normal(1, M, K), normal(2, E, K, std=0.05)
    x[:, 0], W[:, 0] = 1.0, low
    ids, w = w2.moe_route(w2.Router(W, top, score="sigmoid", scale=2.5, n_groups=groups, top_groups=max(1, groups // 2)), x)
    l = f64(x) @ f64(W).T
    assert l.max() < low + 20 and np.ptp(l, axis=1).min() > 1
    got = ids.cpu().numpy().astype(int)
    near(w, renormalised(l, got, 2.5), 2.0 ** -22 * renormalised(l, got, 2.5) + 2.0 ** -149, "weights")
    size = E // groups
    for row, chosen in zip(l, got):                           # the largest ones of the groups with the largest
        best = np.argsort(-row.reshape(groups, size).max(1), kind="stable")[:max(1, groups // 2)]
        free = np.sort((best[:, None] * size + np.arange(size)).ravel())
        assert chosen.tolist() == free[np.argsort(-row[free], kind="stable")[:top]].tolist()


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_a_bias_that_chooses_experts_of_no_weight(w2, score):
    """Experts whose p are 0 in 64 bits, chosen for their bias: the weights are the quotients of their exponentials, without NaN."""
    M, K, E = 7, 256, 72
    x, W = normal(3, M, K), normal(4, E, K, std=0.05)
    x[:, 0] = 1.0
    W[:, 0] = -1000.0
    W[10, 0] = 1000.0                                         # has all of a softmax, and is not chosen
    bias = torch.zeros(E, device="cuda")
    bias[20:24] = torch.tensor([8.0, 7.0, 6.0, 5.0], device="cuda")
    ids, w = w2.moe_route(w2.Router(W, 4, score=score, choice_bias=bias), x)
    assert ids.tolist() == [[20, 21, 22, 23]] * M
    ref = renormalised(f64(x) @ f64(W).T, ids.cpu().numpy().astype(int), 1.0)
    near(w, ref, 2.0 ** -22 * ref, "weights")
    ids, w = w2.moe_route(w2.Router(W, 5, score=score, choice_bias=bias), x)      # the fifth is the one with weight
    assert ids.tolist() == [[20, 21, 22, 23, 10]] * M and w[:, 4].eq(1).all() and not w[:, :4].any()
    ids, w = w2.moe_route(w2.Router(W, 4, score=score, choice_bias=bias, renormalise=False), x)
    assert not w.any()                                        # p itself, which fp32 does not hold


# ------------------------------------------------------------------ between two blocks: rows of more than four vectors a thread
@pytest.mark.gpu
@pytest.mark.parametrize("N", [32776, 40960, 49160, 65528])
@pytest.mark.parametrize("rdt", [torch.float32, torch.bfloat16])
def test_norm_of_wide_rows(w2, N, rdt):
    for post, gate, offset in ((True, "rows", 1.0), (True, "vector", 0.0), (False, "none", 0.5)):
        norm_case(w2, 3, N, rdt, post=post, gate=gate, offset=offset, pad=8, scales=(0.5, 0.22), quantize=N % 256 == 0, seed=N)
        norm_case(w2, 70, N, rdt, post=post, gate=gate, offset=offset, in_place=True, seed=N + 1)
    norm_case(w2, 2, N, rdt, block=False, seed=N + 2)
    norm_case(w2, 2, N, rdt, residual=False, post=True, seed=N + 3)


# ------------------------------------------------------------------ experts: what a row's numbers keep, on each of the three ways through
WAYS = [(4, 2), (80, 64), (300, 2)]                           # rows, experts: two launches, few rows an expert, many


def one_number(w2, E, G, up, down, hidden=256, inter=256):
    """Experts with h = silu(g) u, g = u = up * (a row's first number) in every column, and Y = down * h[0] in every one."""
    codes = np.full((E, hidden, 2 * inter), 2), np.full((E, inter, hidden), 2)
    for c in codes:
        c[:, 0] = 3
    return MadeBank(w2, hidden, inter, G, (codes[0], np.full((E, hidden // G, 2 * inter), up)), (codes[1], np.full((E, inter // G, hidden), down)))


def first_numbers(M, hidden, values):
    x = torch.zeros(M, hidden, dtype=torch.float64)
    x[:, 0] = torch.tensor([values[i % len(values)] for i in range(M)], dtype=torch.float64)
    x = x.bfloat16()
    return x.cuda(), x[:, 0].double().numpy()


def through_one(w2, bank, x, base=None):
    M = x.shape[0]
    ids, weights = torch.zeros(M, 1, dtype=torch.int32, device="cuda"), torch.ones(M, 1, device="cuda")
    return f64(w2.moe_experts(bank.experts, x, ids, weights, base=base))


@pytest.mark.gpu
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("M,E", WAYS)
def test_experts_round_h_by_half_a_step_of_nine_bits(w2, M, E, G):
    """Y's own rounding does not hide h's: base is the negative of the result in bf16, so that what is left (exact in fp32) is their
    difference, which 2^-8 of itself rounds.  h: 2^-9 of it, and 2^-20 for the exponential, the reciprocal and three products in 32 bits."""
    bank = one_number(w2, E, G, 1.0, 1.0)
    values = np.random.default_rng(M + G).uniform(0.25, 4.0, M) * np.random.default_rng(G).choice([-1.0, 1.0], M)
    x, g = first_numbers(M, 256, list(values))
    ref = g / (1.0 + np.exp(-g)) * g
    b = torch.tensor(ref).bfloat16()
    base = -b.cuda()[:, None].repeat(1, 256).contiguous()
    left = (ref - b.double().numpy())[:, None].repeat(256, 1)
    tol = (2.0 ** -9 + 2.0 ** -20) * np.abs(ref)[:, None]
    near(through_one(w2, bank, x, base), left, tol + 2.0 ** -8 * (np.abs(left) + tol), "h")


@pytest.mark.gpu
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("M,E", WAYS)
def test_experts_smallest_numbers(w2, M, E, G):
    """Rows of numbers down to bf16's smallest denormal, met by scales that bring them up: x is exact.  Then an h down to 2^-133: 2^-9 of it
    or 2^-137, half a step of the second part at the smallest power of two.  Y: its rounding, u; 2^-16 for what is done in 32 bits."""
    bank = one_number(w2, E, G, 2.0 ** 100, 2.0 ** 70)
    x, g = first_numbers(M, 256, [2.0 ** -115, -2.0 ** -120, 255 * 2.0 ** -133, 1.5 * 2.0 ** -126, 2.0 ** -126, -2.0 ** -127, 3 * 2.0 ** -129, 2.0 ** -130, 5 * 2.0 ** -133, 2.0 ** -133])
    g = g * 2.0 ** 100
    ref = (g / (1.0 + np.exp(-g)) * g * 2.0 ** 70)[:, None].repeat(256, 1)
    near(through_one(w2, bank, x), ref, (U + U / 2 + 2.0 ** -16) * np.abs(ref), "smallest x")
    bank = one_number(w2, E, G, 1.0, 2.0 ** 100)
    x, g = first_numbers(M, 256, [2.0 ** -57, -2.0 ** -60, 1.375 * 2.0 ** -60, 2.0 ** -62, 1.25 * 2.0 ** -62, 2.0 ** -63, 1.5 * 2.0 ** -64, 2.0 ** -65, -1.5 * 2.0 ** -66])
    h = (g / (1.0 + np.exp(-g)) * g)[:, None].repeat(256, 1)
    ref = h * 2.0 ** 100
    near(through_one(w2, bank, x), ref, (U + 2.0 ** -16) * np.abs(ref) + np.maximum(U / 2 * np.abs(h), 2.0 ** -137) * (1 + U) * 2.0 ** 100, "smallest h")


@pytest.mark.gpu
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("M,E", [(1, 6), (5, 6), (40, 64), (150, 6)])
@pytest.mark.parametrize("f", [1e-16, 1e-18, 1e-30, 1e-37])
def test_experts_rows_of_tiny_numbers(w2, M, E, G, f):
    """Ordinary weights, rows of tiny numbers: finite, and near the definition beside what 32 bits hold of h and bf16 of Y.  Past the usual
    bound: h's 2^-137 times inter * 2 slots * 0.1 (51 of them), half a step of Y's denormals (2^-134) and of 1000 operations' (2^-149): 2^-131."""
    bank = Bank(w2, 512, 256, E, G, seed=E + G)
    x, w = (normal(1, M, 512, dtype=torch.float32) * f).bfloat16(), mixing(M, 2, 2)
    ids = choices(M, E, 2, 3)
    ref, mag, h_err = want.experts(f64(x), ids.cpu().numpy(), f64(w), bank.weights(0), bank.weights(1))
    near(w2.moe_experts(bank.experts, x, ids, w), ref, U * np.abs(ref) + (U + CUT) * mag + CUT * h_err + 2.0 ** -131, f"numbers of {f}")


# ------------------------------------------------------------------ experts: kernels that ordinary sizes do not reach
SPLIT = [(hidden, 256, 16, 8, 11) for hidden in (2048, 2304, 2560, 2816, 3328)] + [(256, inter, 16, 8, 11) for inter in (2048, 2304, 2560, 2816, 3328)] + \
        [(2304, 2560, 12, 7, 10)]
UNITS = [(256, 1024, 64, 8, 4, 2), (512, 1024, 64, 8, 8, 4), (256, 2048, 64, 8, 8, 8), (256, 1536, 64, 8, 6, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("hidden,inter,E,k,M", SPLIT)
def test_experts_few_rows_two_ranges_of_k(w2, G, hidden, inter, E, k, M):
    """K of 8 to 13 tiles in two ranges: even ones, a shorter second one, one to three steps behind the last four."""
    bank = Bank(w2, hidden, inter, E, G, seed=hidden + inter)
    x, w = normal(M, M, hidden), mixing(M, k, M)
    experts_check(w2, bank, x, choices(M, E, k, M), w, what=f"{hidden} x {inter}")
    experts_check(w2, bank, x, choices(M, E, k, M, distinct=False), w, base=normal(2, M, hidden), what=f"{hidden} x {inter}, repeated")


@pytest.mark.gpu
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("hidden,inter,E,k,M,units", UNITS)
def test_experts_several_groups_of_blocks_a_workgroup(w2, G, hidden, inter, E, k, M, units):
    bank = Bank(w2, hidden, inter, E, G, seed=hidden + inter)
    x, w = normal(M, M, hidden), mixing(M, k, M)
    experts_check(w2, bank, x, choices(M, E, k, M), w, what=f"{hidden} x {inter}")
    experts_check(w2, bank, x, choices(M, E, k, M, skew=4.0), w, base=normal(2, M, hidden), what=f"{hidden} x {inter}, skewed")


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,top_groups,top", [(32, 4, 2, 8), (256, 8, 8, 16), (60, 3, 3, 60)])
def test_route_sums_of_groups_leave_the_scores_order(w2, score, E, groups, top_groups, top):
    """Scores of 100 and more apart: sigmoids are 1 and a softmax has one number, so that sums over groups are equal and the lower ones go;
    in them the scores' own order decides."""
    x, W = normal(5, 6, 256), normal(6, E, 256, std=0.2)
    x[:, 0] = 1.0
    W[:, 0] = torch.tensor(np.random.default_rng(E).permutation(E) * 128.0 + 128.0).bfloat16()
    ids, w = w2.moe_route(w2.Router(W, top, score=score, n_groups=groups, top_groups=top_groups, group_top=2), x)
    l, size = f64(x) @ f64(W).T, E // groups
    assert l.min() > 64
    for row, chosen in zip(l, ids.cpu().numpy()):
        p = 1.0 / (1.0 + np.exp(-row)) if score == "sigmoid" else np.exp(row - row.max())
        best = np.sort(p.reshape(groups, size), 1)[:, -2:].sum(1)
        kept = np.argsort(-best, kind="stable")[:top_groups]
        free = np.sort((kept[:, None] * size + np.arange(size)).ravel())
        assert chosen.tolist() == free[np.argsort(-row[free], kind="stable")[:top]].tolist()
    assert torch.isfinite(w).all()


# ------------------------------------------------------------------ between two blocks: int8 rows of numbers that are none
@pytest.mark.gpu
@pytest.mark.parametrize("N", [256, 5120])
def test_norm_quantised_rows_where_numbers_are_not_finite(w2, N):
    """x's int8 rows are those of quantize_rows for rows of NaN, of infinities, of the largest numbers and of denormals too."""
    r = normal(7, 6, N, dtype=torch.float32)
    weight = torch.ones(N, dtype=torch.bfloat16, device="cuda")
    weight[3], weight[9], weight[11] = float("inf"), 3e38, float("nan")
    r[0] *= 1e-38
    r[1] = 0.0
    r[2, 5] = float("nan")
    r[3, 5] = float("inf")
    for w in (None, weight):
        x, _, xq, sx = w2.residual_norm(w2.Norm(w, eps=0.5), r, None, quantize=True)
        bits, scale, _ = w2.quantize_rows(x)
        assert torch.equal(xq, bits) and torch.equal(sx.view(torch.int32), scale.view(torch.int32))
