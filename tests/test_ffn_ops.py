"""The operators of a layer's feed-forward half against their definitions in 64 bits, and their refusals.

Bounds, with u = 2^-8 the relative error of one rounding to bf16 and e = 2^-24 that of fp32:
* residual_norm: r' in fp32 is a sum of two terms of up to three products, one of them by a factor whose sum of squares has at most
  64 terms in a row and 10 levels above them: 2^-17 of the terms' magnitude covers (74 / 2 + 8) e; bf16 adds u of the number.  x the same,
  twice (its own factor and r's error);
* moe_route: scores are sums in 64 bits: wherever two of them are further apart than 2^-40 the choice has to be exact; weights are
  rounded once to fp32 (2 e with the arithmetic before it);
* moe_experts: a matrix instruction cuts each of 8 neighbouring products off 13 bits below the largest one's exponent: 7 * 2^-13 of the sum of
  magnitudes at most, in either product; h is the sum of two numbers of four bits (2^-9 of it) and a row's sums may wait in fp16 (2^-11), together
  less than u; Y is rounded once (u).  By norms: two
  independent roundings whose relative error is at most 2^-8 and, spread evenly over a step, 2^-8 / sqrt(3) in the mean square:
  0.0032 together, 0.0036 with what the products lose.
"""
import ctypes

import numpy as np
import pytest

from oracle import ffn_oracle as want

torch = pytest.importorskip("torch")
U = 2.0 ** -8
CUT = 7 * 2.0 ** -13


@pytest.fixture(scope="module")
def w2():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_06753_amd import binding
    return binding


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def near(got, ref, tol, what):
    got = f64(got) if torch.is_tensor(got) else got
    assert np.isfinite(got).all(), f"{what}: {np.count_nonzero(~np.isfinite(got))} outputs are not finite"
    off = np.abs(got - ref) - tol
    assert (off <= 0).all(), f"{what}: {np.count_nonzero(off > 0)} of {off.size} off, worst by {off.max():.3g} over its bound"


def normal(seed, *shape, dtype=torch.bfloat16, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


# ------------------------------------------------------------------ between two blocks
def norm_case(w2, M, N, rdt=torch.float32, post=False, gate="none", offset=0.0, weight=True, residual=True, block=True, pad=0,
              in_place=False, quantize=False, scales=(1.0, 1.0), seed=0):
    r = normal(seed, M, N + pad, dtype=rdt, std=3.0)[:, :N] if residual else None
    y = normal(seed + 1, M, N + pad)[:, :N] if block else None
    w = (1.0 - offset + normal(seed + 2, N, dtype=torch.float32, std=0.3)).bfloat16() if weight else None
    pw = (1.0 - offset + normal(seed + 3, N, dtype=torch.float32, std=0.3)).bfloat16() if post else None
    g = None if gate == "none" else normal(seed + 4, N) if gate == "vector" else normal(seed + 4, M, N + pad)[:, :N]
    norm = w2.Norm(w, post_weight=pw, weight_offset=offset, eps=1e-5, residual_scale=scales[0], block_scale=scales[1])
    rows = None if g is None else f64(g) if g.dim() == 2 else f64(g)[None]
    x64, r64, rmag, xmag = want.residual_norm(f64(r), f64(y), f64(w), f64(pw), post, rows, offset, 1e-5, *map(np.float32, scales))
    if in_place:
        out, r_out = y, r
    else:
        out = torch.full((M, N + pad), 3.0, dtype=torch.bfloat16, device="cuda")[:, :N]
        r_out = torch.full((M, N + pad), 3.0, dtype=rdt, device="cuda")[:, :N]
    got = w2.residual_norm(norm, r, y, gate=g, out=out, residual_out=r_out, quantize=quantize)
    what = f"residual_norm M={M} N={N} {rdt} post={post} gate={gate}"
    ur = U if rdt is torch.bfloat16 else 0.0
    near(got[1], r64, ur * np.abs(r64) + 2.0 ** -17 * rmag, what + " r'")
    near(got[0], x64, U * np.abs(x64) + 2.0 ** -16 * xmag, what + " x")
    if pad and not in_place:
        assert (out._base[:, N:] == 3.0).all() and (r_out._base[:, N:] == 3.0).all(), "columns past the row's end were written"
    if quantize:
        xq, sx, _ = w2.quantize_rows(got[0])
        assert torch.equal(got[2], xq) and torch.equal(got[3], sx), what + ": not the rows that quantize_rows makes of x"


@pytest.mark.gpu
@pytest.mark.parametrize("N", [8, 64, 504, 520, 2048, 4096, 5128, 8192, 16384, 28672, 65536])
@pytest.mark.parametrize("rdt", [torch.float32, torch.bfloat16])
def test_norm_widths(w2, N, rdt):
    for M in (1, 3, 70):
        norm_case(w2, M if N < 16384 else min(M, 3), N, rdt, post=True, gate="rows", offset=1.0, pad=8, scales=(0.5, 0.22), seed=N + M)
        norm_case(w2, M if N < 16384 else min(M, 3), N, rdt, seed=N + M + 7)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["none", "vector", "rows"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("rdt", [torch.float32, torch.bfloat16])
def test_norm_forms(w2, gate, post, rdt):
    norm_case(w2, 5, 768, rdt, post=post, gate=gate, in_place=True, seed=1)
    norm_case(w2, 300, 512, rdt, post=post, gate=gate, weight=False, seed=2)
    norm_case(w2, 4, 1280, rdt, post=post, gate=gate, residual=False, seed=3)
    norm_case(w2, 4, 1280, rdt, block=False, seed=4, scales=(0.7, 1.0))


@pytest.mark.gpu
def test_norm_more_rows_than_a_launch_takes(w2):
    norm_case(w2, 2 ** 20 + 5, 8, gate="rows", post=True, seed=5)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(1, 256), (3, 4096), (90, 5120), (2, 65536), (2, 16)])
def test_norm_quantised_rows_are_those_of_quantize_rows(w2, M, N):
    if N % 256 == 0:                                          # what quantize_rows takes
        norm_case(w2, M, N, post=True, gate="vector", quantize=True, seed=N)
    x = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    x2, r, xq, sx = w2.residual_norm(w2.Norm(), x, x.clone(), quantize=True)
    assert not x2.any() and not r.any() and not xq.any() and not sx.any()      # rows of zeros stay zeros


@pytest.mark.gpu
def test_norm_of_the_last_block_and_of_none(w2):
    """Only the residual, only x, only int8 rows: through the C entry; a NaN stays in its row."""
    lib, M, N = w2.raw(), 3, 512
    r, y = normal(1, M, N, dtype=torch.float32), normal(2, M, N)
    w = torch.ones(N, dtype=torch.bfloat16, device="cuda")
    x, r2 = w2.residual_norm(w2.Norm(w, post_weight=w, eps=0.0), r, None)       # no block: zero, not 0 / 0
    assert torch.equal(r2, r) and torch.isfinite(x).all()
    norm = w2.Norm(block_scale=0.5)
    x, r2, xq, sx = w2.residual_norm(norm, r, y, quantize=True)
    s = torch.cuda.current_stream().cuda_stream
    only = torch.zeros_like(r)
    assert lib.w2_residual_norm(norm._ref, r.data_ptr(), 0, N, y.data_ptr(), N, M, N, only.data_ptr(), N, None, 0, None, None, s) == 0
    assert torch.equal(only, r2)
    ox = torch.zeros_like(x)
    assert lib.w2_residual_norm(norm._ref, r.data_ptr(), 0, N, y.data_ptr(), N, M, N, None, 0, ox.data_ptr(), N, None, None, s) == 0
    assert torch.equal(ox, x)
    oq, osx = torch.zeros_like(xq), torch.zeros_like(sx)
    assert lib.w2_residual_norm(norm._ref, r.data_ptr(), 0, N, y.data_ptr(), N, M, N, None, 0, None, 0, oq.data_ptr(), osx.data_ptr(), s) == 0
    assert torch.equal(oq, xq) and torch.equal(osx, sx)
    y[1, 5] = float("nan")
    x3, r3 = w2.residual_norm(norm, r, y)
    assert torch.isnan(x3[1]).all() and torch.equal(x3[0], x[0]) and torch.equal(x3[2], x[2]) and torch.isnan(r3[1]).sum() == 1


# ------------------------------------------------------------------ the router
def route_case(w2, M, K, E, top, seed=0, pad=0, std=1.5, **kw):
    x = normal(seed, M, K + pad)[:, :K]
    W = normal(seed + 1, E, K + pad, std=std / K ** 0.5)[:, :K]
    bias = normal(seed + 2, E, dtype=torch.float32, std=0.1) if kw.pop("bias", False) else None
    router = w2.Router(W, top, choice_bias=bias, **kw)
    ids64, w64, l64, gaps = want.route(f64(x), f64(W), top, choice_bias=f64(bias), **kw)
    ws = torch.full((w2.moe_route_workspace_size(router, M),), 0xff, dtype=torch.uint8, device="cuda")
    logits = torch.empty(M, E, dtype=torch.float32, device="cuda")
    ids, w = w2.moe_route(router, x, logits=logits, workspace=ws)
    clear = gaps > 2.0 ** -40
    what = f"route M={M} K={K} E={E} top={top} {kw}"
    assert clear.mean() > 0.99, what
    assert np.array_equal(ids.cpu().numpy()[clear], ids64[clear]), what
    near(f64(w)[clear], w64[clear], 2.0 ** -23 * np.abs(w64[clear]), what)
    near(logits, l64, 2.0 ** -24 * np.abs(l64) + 2.0 ** -40, what + " logits")
    return ids, w


@pytest.mark.gpu
@pytest.mark.parametrize("E,top", [(1, 1), (2, 2), (8, 2), (60, 4), (64, 6), (65, 8), (128, 8), (160, 6), (256, 8), (300, 64),
                                   (512, 10), (1024, 16)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_sizes(w2, E, top, score):
    for M in (1, 9, 67):
        route_case(w2, M, 512, E, top, score=score, seed=E + M)
    route_case(w2, 5, 1032, E, top, score=score, renormalise=False, scale=2.5, bias=True, pad=8, seed=E)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2, 7, 8, 15, 16, 17, 33, 64, 65, 200, 1000])
@pytest.mark.parametrize("K", [8, 256, 2048, 4104])
def test_route_row_counts(w2, M, K):
    route_case(w2, M, K, 72, 5, seed=M + K)


@pytest.mark.gpu
@pytest.mark.parametrize("M,E", [(2100, 72), (200, 1000)])   # enough tiles of 32 x 32 that K stays in one part
@pytest.mark.parametrize("K", [8, 32, 72, 264, 1000, 4104])
def test_route_many_rows(w2, M, E, K):
    route_case(w2, M, K, E, 5, seed=M + K)


@pytest.mark.gpu
@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,top_groups,top", [(32, 8, 3, 8), (60, 4, 2, 5), (256, 8, 4, 8), (160, 8, 3, 6), (64, 64, 5, 5),
                                                     (1024, 4, 1, 16), (40, 2, 2, 9)])
def test_route_groups(w2, group_top, bias, score, E, groups, top_groups, top):
    route_case(w2, 33, 384, E, top, score=score, bias=bias, n_groups=groups, top_groups=top_groups, group_top=group_top, seed=E + top)


@pytest.mark.gpu
def test_route_ties_saturation_and_numbers_that_are_none(w2):
    K, E = 256, 64
    x = normal(1, 6, K)
    W = normal(2, E, K)
    W[40] = W[7]                                             # equal scores: the lower index first
    W[63] = W[7]
    ids, _ = w2.moe_route(w2.Router(W, E), x)
    for row in ids.tolist():
        assert sorted(row) == list(range(E)) and row.index(40) == row.index(7) + 1 and row.index(63) == row.index(7) + 2
    ids, w = w2.moe_route(w2.Router(W, 3), torch.zeros_like(x))
    assert ids.tolist() == [[0, 1, 2]] * 6 and torch.allclose(w, torch.full_like(w, 1 / 3))
    # scores so far apart that probabilities are 0 or 1: the scores' own order still decides
    ids64 = np.argsort(-(f64(x) @ f64(W[:40]).T), axis=1, kind="stable")[:, :5]
    for score in ("softmax", "sigmoid"):
        ids, w = w2.moe_route(w2.Router((W[:40].float() * 128).bfloat16(), 5, score=score), x)
        assert np.array_equal(ids.cpu().numpy(), ids64) and torch.isfinite(w).all()
    # a NaN counts as lower than any number, and ids stay distinct and inside
    W[3, 0] = float("nan")
    ids, _ = w2.moe_route(w2.Router(W, E), x)
    assert all(sorted(r) == list(range(E)) and r[-1] == 3 for r in ids.tolist())
    x[2, 9] = float("nan")
    ids, _ = w2.moe_route(w2.Router(W, 5), x)
    assert ids[2].tolist() == [0, 1, 2, 3, 4]


# ------------------------------------------------------------------ experts
class Bank:
    """Experts with their codes: blobs for the library, weights in 64 bits for the oracle."""

    def __init__(self, w2, hidden, inter, E, G, codec=0, seed=0, pad=0):
        rng = np.random.default_rng(seed)
        self.hidden, self.inter, self.E, self.G, self.zero = hidden, inter, E, G, 2 if codec == 0 else 1
        self.parts, blobs = [], []
        for K, N in ((hidden, 2 * inter), (inter, hidden)):
            codes = rng.integers(0, 4 if codec == 0 else 3, (E, K, N), dtype=np.uint8)
            scales = torch.tensor(rng.uniform(0.005, 0.05, (E, K // G, N)), dtype=torch.float32).bfloat16()
            size = w2.packed_size(K, N, G)
            blob = torch.full((E, size + pad), 0xff, dtype=torch.uint8, device="cuda")
            for e in range(E):
                blob[e, :size] = w2.prepack(torch.from_numpy(codes[e]).cuda(), scales[e].cuda(), G, codec)
            self.parts.append((codes, scales.double().numpy()))
            blobs.append(blob)
        self.experts = w2.Experts(*blobs, hidden=hidden, inter=inter, G=G)

    def weights(self, part):
        codes, scales = self.parts[part]
        return lambda e: want.dequantise(codes[e], scales[e], self.G, self.zero) if 0 <= e < self.E else None


def experts_check(w2, bank, x, ids, weights, base=None, out=None, what="experts", workspace=None):
    M, k = ids.shape
    ref, mag, h_err = want.experts(f64(x), ids.cpu().numpy(), f64(weights), bank.weights(0), bank.weights(1), f64(base))
    if workspace is None:
        workspace = torch.full((w2.moe_experts_workspace_size(bank.experts, M, k),), 0xff, dtype=torch.uint8, device="cuda")
    y = w2.moe_experts(bank.experts, x, ids, weights, base=base, out=out, workspace=workspace)
    near(y, ref, U * np.abs(ref) + (U + CUT) * mag + CUT * h_err, what)
    norm = np.linalg.norm(ref)
    assert np.linalg.norm(f64(y) - ref) <= 0.0036 * norm + 1e-30, f"{what}: {np.linalg.norm(f64(y) - ref) / norm:.4f} off"
    return y


def choices(M, E, k, seed, skew=0.0, distinct=True):
    rng = np.random.default_rng(seed)
    if not distinct:
        return torch.tensor(rng.integers(0, E, (M, k)), dtype=torch.int32, device="cuda")
    score = rng.gumbel(size=(M, E)) - skew * np.log1p(np.arange(E))
    return torch.tensor(np.argsort(-score, 1)[:, :k].copy(), dtype=torch.int32, device="cuda")


def mixing(M, k, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.rand(M, k, generator=g).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2, 3, 7, 8, 9, 16, 17, 31, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("G", [64, 128])
def test_experts_row_counts(w2, M, G):
    bank = Bank(w2, 512, 256, 12, G, seed=G)
    x, w = normal(M, M, 512), mixing(M, 4, M)
    experts_check(w2, bank, x, choices(M, 12, 4, M), w, what=f"M={M} G={G}")
    experts_check(w2, bank, x, choices(M, 12, 4, M + 1, skew=3.0), w, base=normal(M + 2, M, 512), what=f"M={M} G={G} skewed")


@pytest.mark.gpu
@pytest.mark.parametrize("hidden,inter,E,k", [(256, 256, 1, 1), (256, 512, 3, 3), (768, 256, 40, 1), (1280, 512, 9, 5), (2048, 768, 8, 2),
                                              (256, 2304, 2, 2), (4096, 256, 4, 2), (512, 4096, 3, 2)])
@pytest.mark.parametrize("codec", [0, 1])
def test_experts_shapes(w2, hidden, inter, E, k, codec):
    bank = Bank(w2, hidden, inter, E, 128 if codec else 64, codec, seed=hidden + inter, pad=48)
    for M in (1, 6, 40, 150):
        experts_check(w2, bank, normal(M, M, hidden), choices(M, E, k, M, skew=0.5), mixing(M, k, M),
                      what=f"hidden={hidden} inter={inter} E={E} k={k} M={M}")


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 60, 270])
def test_experts_dropped_repeated_and_strided(w2, M):
    bank = Bank(w2, 512, 512, 10, 128, seed=3)
    wide = normal(1, M, 520)
    x, w = wide[:, :512], mixing(M, 6, 2)
    ids = choices(M, 10, 6, 4, distinct=False)                # the same expert in several slots of a row
    ids[:, 2] = -1
    ids[0] = torch.tensor([-1, 10, -5, 2 ** 31 - 1, -2 ** 31, 1000], dtype=torch.int32)      # a row without experts
    w[:, 2] = float("nan")                                    # weights of no expert are not read
    w[0] = float("inf")
    base = normal(5, M, 528)[:, :512]
    clean = torch.where((ids >= 0) & (ids < 10), w, torch.zeros_like(w))
    ref, mag, h_err = want.experts(f64(x), ids.cpu().numpy(), f64(clean), bank.weights(0), bank.weights(1), f64(base))
    out = torch.full((M, 536), 3.0, dtype=torch.bfloat16, device="cuda")[:, :512]
    y = w2.moe_experts(bank.experts, x, ids, w, base=base, out=out)
    near(y, ref, U * np.abs(ref) + (U + CUT) * mag + CUT * h_err, "dropped and repeated")
    assert torch.equal(y[0], base[0])                         # base alone, unchanged
    assert (out._base[:, 512:] == 3.0).all(), "columns past the row's end were written"
    z = w2.moe_experts(bank.experts, x, ids, w)
    assert not z[0].any()                                     # and zero without a base
    same = base.clone() if base.is_contiguous() else base.contiguous()
    again = w2.moe_experts(bank.experts, x, ids, w, base=same, out=same)
    assert again is same and torch.equal(again, y)            # in place


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 4, 33, 200])
def test_experts_rows_do_not_meet(w2, M):
    """All rows to one expert and back; what a row gives does not depend on the other rows, NaN and infinities among them."""
    bank = Bank(w2, 512, 256, 6, 64, seed=5)
    x, w = normal(1, M, 512), mixing(M, 2, 2)
    ids = torch.full((M, 2), 3, dtype=torch.int32, device="cuda")
    first = experts_check(w2, bank, x, ids, w, what="one expert")
    bad = x.clone()
    bad[M // 2, 100] = float("nan")
    y = w2.moe_experts(bank.experts, bad, ids, w)
    keep = torch.arange(M, device="cuda") != M // 2
    assert torch.equal(y[keep], first[keep]) and torch.isnan(y[M // 2]).all()
    bad[M // 2, 100] = float("inf")
    y = w2.moe_experts(bank.experts, bad, ids, w)
    assert torch.equal(y[keep], first[keep]) and not torch.isfinite(y[M // 2]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 40, 150])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_experts_scales_that_are_no_numbers_stay_in_their_columns(w2, M, bad):
    bank = Bank(w2, 512, 256, 6, 128, seed=7)
    x, w, ids = normal(1, M, 512), mixing(M, 2, 2), choices(M, 6, 2, 3)
    good = w2.moe_experts(bank.experts, x, ids, w).clone()
    codes, scales = bank.parts[1]
    e = int(ids[0, 0])
    s = torch.from_numpy(scales[e]).bfloat16()
    s[:, 5] = bad
    down = bank.experts.down.clone()
    size = w2.packed_size(256, 512, 128)
    down[e, :size] = w2.prepack(torch.from_numpy(codes[e]).cuda(), s.cuda(), 128, 0)
    y = w2.moe_experts(w2.Experts(bank.experts.gate_up, down, hidden=512, inter=256, G=128), x, ids, w)
    hit = (ids == e).any(1)
    assert not torch.isfinite(y[hit, 5]).any()
    y[:, 5] = good[:, 5]
    assert torch.equal(y, good)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 40, 150])
def test_experts_numbers_of_every_size(w2, M):
    """Rows of zeros, of tiny and huge numbers, and outliers beside ordinary ones."""
    bank = Bank(w2, 512, 256, 6, 128, seed=6)
    x, w = normal(1, M, 512, dtype=torch.float32), mixing(M, 2, 2)
    x[:, 7] *= 500.0
    x[:, 300:310] *= 1e-4
    ids = choices(M, 6, 2, 3)
    experts_check(w2, bank, x.bfloat16(), ids, w, what="outliers")
    for f in (1e-30, 1e-12, 1e12):                           # z^2 in 32 bits
        experts_check(w2, bank, (x * f).bfloat16(), ids, w, what=f"numbers of {f}") if f > 1e-20 else \
            w2.moe_experts(bank.experts, (x * f).bfloat16(), ids, w)
    y = w2.moe_experts(bank.experts, torch.zeros_like(x).bfloat16(), ids, w)
    assert not y.any()


@pytest.mark.gpu
def test_experts_more_rows_than_go_together(w2):
    """Rows whose parts pass 2 GiB go in turns; offsets of x and Y pass 32 bits.  A row's bits are those of a small batch."""
    M, most = 2 ** 22 + 90, 2 ** 22                          # 512 bytes of a row's two parts in 2 GiB
    bank = Bank(w2, 256, 256, 5, 128, seed=8)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(M, 264, generator=g, device="cuda", dtype=torch.bfloat16)[:, :256]
    ids = torch.randint(-1, 5, (M, 1), generator=g, device="cuda", dtype=torch.int32)
    w = torch.rand(M, 1, generator=g, device="cuda")
    y = w2.moe_experts(bank.experts, x, ids, w)
    for part in (slice(0, 400), slice(most - 400, most), slice(most, M)):
        small = experts_check(w2, bank, x[part].contiguous(), ids[part].contiguous(), w[part].contiguous(), what=str(part))
        assert torch.equal(y[part], small)


@pytest.mark.gpu
def test_experts_larger_workspace_streams_and_graphs(w2):
    """A workspace of the largest batch serves all; a captured call gives the eager one's bits at every replay, with other work
    between them; calls on two streams with workspaces of their own."""
    bank = Bank(w2, 768, 512, 16, 128, seed=7)
    ws = torch.full((w2.moe_experts_workspace_size(bank.experts, 300, 4),), 0xff, dtype=torch.uint8, device="cuda")
    calls = []
    for M in (300, 1, 20, 90):
        x, ids, w = normal(M, M, 768), choices(M, 16, 4, M), mixing(M, 4, M)
        experts_check(w2, bank, x, ids, w, workspace=ws, what=f"M={M} in a larger workspace")
        calls.append((x, ids, w, w2.moe_experts(bank.experts, x, ids, w, workspace=ws).clone(), torch.empty_like(x)))
    for x, ids, w, y, out in calls:
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            w2.moe_experts(bank.experts, x, ids, w, out=out, workspace=ws)
        torch.cuda.current_stream().wait_stream(side)
        with torch.cuda.graph(graph):
            w2.moe_experts(bank.experts, x, ids, w, out=out, workspace=ws)
        for _ in range(3):
            out.fill_(7.0)
            ws.fill_(0xff)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, y)
            (x.float() @ x.float().t()).sum().item()
    streams = [torch.cuda.Stream() for _ in calls]
    spaces = [torch.empty_like(ws) for _ in calls]
    torch.cuda.synchronize()
    for _ in range(3):
        for (x, ids, w, _, out), s, space in zip(calls, streams, spaces):
            with torch.cuda.stream(s):
                w2.moe_experts(bank.experts, x, ids, w, out=out, workspace=space)
    torch.cuda.synchronize()
    for _, _, _, y, out in calls:
        assert torch.equal(out, y)


@pytest.mark.gpu
def test_norm_and_route_in_a_graph(w2):
    x, r, W = normal(1, 50, 1024), normal(2, 50, 1024, dtype=torch.float32), normal(3, 64, 1024, std=0.05)
    norm, router = w2.Norm((1 + normal(4, 1024, std=0.1).float()).bfloat16()), w2.Router(W, 6)
    space = torch.empty(w2.moe_route_workspace_size(router, 50), dtype=torch.uint8, device="cuda")
    x1, r1 = w2.residual_norm(norm, r, x)
    ids1, w1 = w2.moe_route(router, x1, workspace=space)
    out = torch.empty_like(x1), torch.empty_like(r1), torch.empty_like(ids1), torch.empty_like(w1)

    def both():
        w2.residual_norm(norm, r, x, out=out[0], residual_out=out[1])
        w2.moe_route(router, out[0], ids=out[2], weights=out[3], workspace=space)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in out:
            t.zero_()
        space.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, (x1, r1, ids1, w1)):
            assert torch.equal(a, b)


# ------------------------------------------------------------------ the operators together
def layer_and_cache(w2, shared=True, seed=0):
    from paper_2508_06753_amd import attention_block as ab, decoder_layer as dl, synth
    hidden, n_q, n_kv, D, G = 512, 4, 2, 64, 64
    width = (n_q + 2 * n_kv) * D

    def packed(K, N, s):
        codes, scales = synth.make_weights(K, N, G, 0, seed=s)
        return codes, scales, w2.prepack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales.view(np.int16)).cuda(), G)

    bank = Bank(w2, hidden, 256, 12, G, seed=seed + 3)
    one = [packed(hidden, 512, seed + 4), packed(256, hidden, seed + 5)] if shared else None
    attention = ab.AttentionBlock(packed(hidden, width, seed + 1)[2], packed(n_q * D, hidden, seed + 2)[2], hidden, n_q, n_kv, D, G, w2.Rope(D))
    router = w2.Router(normal(seed + 6, 12, hidden, std=0.1), 3, scale=1.5)
    weight = lambda s: (1 + normal(s, hidden, dtype=torch.float32, std=0.2)).bfloat16()  # noqa: E731
    norms = w2.Norm(weight(seed + 7)), w2.Norm(weight(seed + 8), post_weight=weight(seed + 9), block_scale=0.5)
    layer = dl.DecoderLayer(attention, dl.MoeBlock(router, bank.experts, None if one is None else (one[0][2], one[1][2], 256)), *norms)
    k = normal(seed + 10, 24, 16, n_kv, D)
    return ab, layer, bank, one, w2.KVCache(k, torch.zeros_like(k))


@pytest.mark.gpu
@pytest.mark.parametrize("shared", [False, True])
def test_layer_runs_prompts_and_tokens(w2, shared):
    """A step of a layer against the operators' definitions, around the attention that the library computes."""
    ab, layer, bank, one, cache = layer_and_cache(w2, shared)
    table = torch.arange(20, dtype=torch.int32).flip(0).view(2, 10).contiguous().cuda()
    lens = [45, 70]
    for batch in (ab.causal_batch([0, 0], lens, table, 16, "cuda"), ab.causal_batch(lens, [1, 1], table, 16, "cuda")):
        M = batch.positions.shape[0]
        r, y = normal(M, M, 512, dtype=torch.float32), normal(M + 1, M, 512)
        keep = cache.k.clone(), cache.v.clone()
        r2, y2 = layer.step(r.clone(), y, cache, batch)
        cache.k.copy_(keep[0])
        cache.v.copy_(keep[1])
        n1, n2 = layer.attention_norm, layer.moe_norm
        x64, r64, _, _ = want.residual_norm(f64(r), f64(y), f64(n1.weight))
        x = torch.tensor(x64).bfloat16().cuda()
        a = f64(layer.attention.step(x, cache, batch))
        x64, r64, _, _ = want.residual_norm(r64, a, f64(n2.weight), f64(n2.post_weight), True, block_scale=0.5)
        x = f64(torch.tensor(x64).bfloat16())
        router = layer.moe.router
        ids, weights, _, gaps = want.route(x, f64(router.weight), 3, scale=1.5)
        base = None
        if shared:
            (c1, s1, _), (c2, s2, _) = one
            from paper_2508_06753_amd.synth import bf16_bits_to_f32
            w1 = want.dequantise(c1, bf16_bits_to_f32(s1).astype(np.float64), 64, 2)
            wd = want.dequantise(c2, bf16_bits_to_f32(s2).astype(np.float64), 64, 2)
            base, _, _ = want.experts(x, np.zeros((M, 1), int), np.ones((M, 1)), lambda e: w1, lambda e: wd)
        ref, _, _ = want.experts(x, ids, weights, bank.weights(0), bank.weights(1), base)
        assert np.abs(f64(r2) - r64).max() < 0.02 * np.abs(r64).max()
        # a bf16 number rounded the other way somewhere moves what follows, now and then the choice: rows whose choice was clear
        off = np.linalg.norm(f64(y2) - ref, axis=1) / np.linalg.norm(ref, axis=1)
        assert (gaps > 0.01).sum() >= 1 and off[gaps > 0.01].max() < 0.03, off


@pytest.mark.gpu
def test_layer_in_a_graph_and_main(w2, capsys):
    """A captured step of a layer gives the eager one's bits at every replay; the steps of the command are sound."""
    ab, layer, _, _, cache = layer_and_cache(w2)
    table = torch.arange(20, dtype=torch.int32).view(2, 10).contiguous().cuda()
    layer.step(normal(1, 25, 512, dtype=torch.float32), None, cache, ab.causal_batch([0, 0], [20, 5], table, 16, "cuda"))
    batch = ab.causal_batch([20, 5], [1, 3], table, 16, "cuda")
    r, y = normal(2, 4, 512), normal(3, 4, 512)                # a residual of 16 bits
    want_r, want_y = (t.clone() for t in layer.step(r, y, cache, batch))
    space = torch.empty(layer.workspace_size(4, batch, cache), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got_r, got_y = layer.step(r, y, cache, batch, workspace=space)
    for _ in range(3):
        got_r.zero_()
        got_y.zero_()
        space.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got_r, want_r) and torch.equal(got_y, want_y)
        (y.float() @ y.float().t()).sum().item()
    with pytest.raises(ValueError):
        layer.moe.step(y, workspace=space[:64])
    from paper_2508_06753_amd import decoder_layer
    assert decoder_layer.main()
    assert capsys.readouterr().out.count("finite True") == 2


# ------------------------------------------------------------------ refusals
def test_c_entries_refuse_bad_arguments_before_any_launch():
    from paper_2508_06753_amd import binding as w2
    lib, size = w2.raw(), ctypes.c_size_t(0)
    p = 1 << 20                                               # aligned, never read: every call below is refused or has no rows
    F, I = ctypes.c_float, w2.ERR_INVALID_ARG
    SHAPE, ALIGN, SMALL = w2.ERR_UNSUPPORTED_SHAPE, w2.ERR_MISALIGNED, w2.ERR_BUFFER_TOO_SMALL

    def norm(rc, M=2, N=64, dt=0, r=p, ldr=64, y=p, ldy=64, ro=p, ldro=64, x=p, ldx=64, xq=None, sx=None, **kw):
        f = dict(weight=None, post_weight=None, gate=None, ld_gate=0, weight_offset=0.0, eps=1e-6, residual_scale=1.0, block_scale=1.0, post_norm=0)
        f.update(kw)
        s = w2._NormStruct(*[f[n] for n, _ in w2._NormStruct._fields_])
        assert lib.w2_residual_norm(ctypes.byref(s), r, dt, ldr, y, ldy, M, N, ro, ldro, x, ldx, xq, sx, None) == rc, kw or (M, N)

    norm(0, M=0)
    for rc, kw in [(I, dict(M=-1)), (I, dict(N=0)), (SHAPE, dict(N=60)), (SHAPE, dict(N=65544)), (I, dict(dt=2)), (I, dict(eps=-1.0)),
                   (I, dict(eps=float("nan"))), (I, dict(residual_scale=float("inf"))), (I, dict(r=None, y=None)),
                   (I, dict(x=None, ro=None)), (I, dict(xq=p)), (I, dict(sx=p)), (SHAPE, dict(N=72, xq=p, sx=p, ldr=72, ldy=72, ldro=72, ldx=72)),
                   (ALIGN, dict(r=p + 8)), (ALIGN, dict(y=p + 2)), (ALIGN, dict(x=p + 4)), (ALIGN, dict(ro=p + 4)), (ALIGN, dict(weight=p + 2)),
                   (ALIGN, dict(gate=p + 2)), (ALIGN, dict(ldr=60)), (ALIGN, dict(ldy=56)), (ALIGN, dict(ldx=68)), (ALIGN, dict(ldro=0)),
                   (ALIGN, dict(gate=p, ld_gate=8)), (ALIGN, dict(gate=p, ld_gate=68)), (ALIGN, dict(xq=p, sx=p + 2)),
                   (I, dict(ldro=72, x=p + 16)), (I, dict(ldx=72, ro=p + 16))]:
        norm(rc, **kw)
    assert lib.w2_residual_norm(None, p, 0, 64, p, 64, 1, 64, p, 64, p, 64, None, None, None) == I

    def route(rc, M=2, K=64, x=p, ldx=64, ids=p, weights=p, logits=None, ws=p, wb=1 << 30, **kw):
        f = dict(weight=p, choice_bias=None, ldw=64, n_experts=16, top_k=4, score=0, renormalise=1, n_groups=1, top_groups=1, group_top=1, scale=1.0)
        f.update(kw)
        s = w2._RouterStruct(*[f[n] for n, _ in w2._RouterStruct._fields_])
        assert lib.w2_moe_route(ctypes.byref(s), x, ldx, M, K, ids, weights, logits, ws, wb, None) == rc, kw or (M, K)

    route(0, M=0)
    for rc, kw in [(I, dict(M=-1)), (I, dict(K=0)), (SHAPE, dict(K=60)), (SHAPE, dict(M=(1 << 24) + 1)), (I, dict(n_experts=0)), (I, dict(top_k=0)),
                   (SHAPE, dict(n_experts=1025)), (SHAPE, dict(top_k=65, n_experts=128)), (I, dict(score=2)), (I, dict(n_groups=3)), (I, dict(n_groups=0)),
                   (I, dict(n_groups=4, top_groups=5)), (I, dict(top_groups=0)), (I, dict(group_top=3)), (I, dict(top_k=17)),
                   (I, dict(n_groups=8, top_groups=1, top_k=3)), (I, dict(scale=float("nan"))), (I, dict(x=None)), (I, dict(ids=None)),
                   (I, dict(weights=None)), (I, dict(weight=None)), (ALIGN, dict(x=p + 2)), (ALIGN, dict(weight=p + 8)), (ALIGN, dict(ws=p + 8)),
                   (ALIGN, dict(ids=p + 2)), (ALIGN, dict(logits=p + 1)), (ALIGN, dict(choice_bias=p + 2)), (ALIGN, dict(ldx=60)), (ALIGN, dict(ldw=56)),
                   (SMALL, dict(ws=None)), (SMALL, dict(wb=8))]:
        route(rc, **kw)
    assert lib.w2_moe_route(None, p, 64, 1, 64, p, p, None, p, 1 << 30, None) == I
    assert lib.w2_moe_route_workspace_size(None, 1, 64, ctypes.byref(size)) == I

    def experts(rc, M=2, x=p, ldx=256, ids=p, weights=p, k=2, base=None, ldb=256, Y=p + 4096, ldy=256, ws=p, wb=1 << 30, **kw):
        f = dict(gate_up=p, down=p, gate_up_stride=1 << 18, down_stride=1 << 18, hidden=256, inter=256, n_experts=4, G=128)
        f.update(kw)
        s = w2._ExpertsStruct(*[f[n] for n, _ in w2._ExpertsStruct._fields_])
        assert lib.w2_moe_experts(ctypes.byref(s), x, ldx, M, ids, weights, k, base, ldb, Y, ldy, ws, wb, None) == rc, kw or (M, k)

    experts(0, M=0)
    for rc, kw in [(I, dict(M=-1)), (I, dict(k=0)), (SHAPE, dict(k=65)), (I, dict(n_experts=0)), (SHAPE, dict(n_experts=1025)), (I, dict(G=32)),
                   (SHAPE, dict(hidden=128)), (SHAPE, dict(inter=320)), (I, dict(hidden=0)), (SHAPE, dict(hidden=(1 << 17) + 256)),
                   (SHAPE, dict(M=1 << 24)), (I, dict(x=None)), (I, dict(ids=None)), (I, dict(weights=None)), (I, dict(Y=None)), (I, dict(gate_up=None)),
                   (I, dict(down=None)), (ALIGN, dict(x=p + 2)), (ALIGN, dict(Y=p + 8)), (ALIGN, dict(base=p + 8)), (ALIGN, dict(gate_up=p + 8)),
                   (ALIGN, dict(ws=p + 8)), (ALIGN, dict(ids=p + 2)), (ALIGN, dict(weights=p + 1)), (ALIGN, dict(ldx=248)), (ALIGN, dict(ldy=260)),
                   (ALIGN, dict(base=p, ldb=0)), (I, dict(Y=p)), (I, dict(base=p + 4096, ldb=264)), (ALIGN, dict(gate_up_stride=(1 << 18) + 8)),
                   (SMALL, dict(gate_up_stride=1 << 12)), (SMALL, dict(down_stride=1 << 12)), (SMALL, dict(ws=None)), (SMALL, dict(wb=16))]:
        experts(rc, **kw)
    assert lib.w2_moe_experts(None, p, 256, 1, p, p, 1, None, 256, p, 256, p, 1 << 30, None) == I
    assert lib.w2_moe_experts_workspace_size(None, 1, 1, ctypes.byref(size)) == I


def test_workspaces_grow_with_the_batch():
    """The size for a program's largest batch serves every smaller one."""
    from paper_2508_06753_amd import binding as w2
    lib, size = w2.raw(), ctypes.c_size_t(0)
    for hidden, inter, E, k in [(256, 256, 1, 1), (4096, 1024, 128, 8), (4096, 14336, 8, 2), (2048, 768, 64, 6), (1 << 17, 256, 1024, 3)]:
        s = w2._ExpertsStruct(None, None, 0, 0, hidden, inter, E, 128)
        last = 0
        for M in list(range(1, 200)) + [255, 256, 257, 1000, 4096, 1 << 18]:
            assert lib.w2_moe_experts_workspace_size(ctypes.byref(s), M, k, ctypes.byref(size)) == 0
            assert size.value >= last, (hidden, inter, E, k, M)
            last = size.value
    for E in (1, 64, 1000):
        s = w2._RouterStruct(None, None, 64, E, 1, 0, 1, 1, 1, 1, 1.0)
        last = 0
        for M in list(range(1, 200)) + [255, 256, 257, 1000, 4096, 1 << 18]:
            assert lib.w2_moe_route_workspace_size(ctypes.byref(s), M, 4096, ctypes.byref(size)) == 0
            assert size.value >= last
            last = size.value


@pytest.mark.gpu
def test_binding_refuses_bad_tensors(w2):
    x, r = normal(1, 4, 256), normal(2, 4, 256, dtype=torch.float32)
    w = normal(3, 256)
    for call in [lambda: w2.Norm(w[None]), lambda: w2.Norm(w.float()), lambda: w2.Norm(w, w[:128]), lambda: w2.Norm(w, w, post_norm=False),
                 lambda: w2.Norm(w.cpu()), lambda: w2.residual_norm(w2.Norm(w[:128]), r, x), lambda: w2.residual_norm(w2.Norm(w), None, None),
                 lambda: w2.residual_norm(w2.Norm(w), r[:2], x), lambda: w2.residual_norm(w2.Norm(w), r.half(), x),
                 lambda: w2.residual_norm(w2.Norm(w), r, x.float()), lambda: w2.residual_norm(w2.Norm(w), r, x, gate=w[:64]),
                 lambda: w2.residual_norm(w2.Norm(w), r, x, gate=r), lambda: w2.residual_norm(w2.Norm(w), r, x, out=x[:2]),
                 lambda: w2.residual_norm(w2.Norm(w), r, x, residual_out=x), lambda: w2.residual_norm(w2.Norm(w), r.t(), x.t()),
                 lambda: w2.Router(w, 1), lambda: w2.Router(x.float(), 1), lambda: w2.Router(x, 1, score="top"),
                 lambda: w2.Router(x, 1, choice_bias=r[0])]:
        with pytest.raises(ValueError):
            call()
    router = w2.Router(normal(4, 8, 256), 2)
    i32, f32 = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    for call in [lambda: w2.moe_route(router, x[:, :128]), lambda: w2.moe_route(router, r), lambda: w2.moe_route(router, x, ids=i32[:2]),
                 lambda: w2.moe_route(router, x, weights=i32), lambda: w2.moe_route(router, x, logits=f32)]:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(w2.W2Error):
        w2.moe_route(router, x, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(w2.W2Error):
        w2.moe_route(w2.Router(normal(4, 8, 256), 9), x)
    bank = Bank(w2, 256, 256, 2, 128)
    gu, dn = bank.experts.gate_up, bank.experts.down
    for call in [lambda: w2.Experts(gu[0], dn, 256, 256, 128), lambda: w2.Experts(gu[:, :64], dn, 256, 256, 128), lambda: w2.Experts(gu, dn[:1], 256, 256, 128),
                 lambda: w2.Experts(gu.cpu(), dn, 256, 256, 128), lambda: w2.moe_experts(bank.experts, r, i32, f32),
                 lambda: w2.moe_experts(bank.experts, x, i32[0], f32), lambda: w2.moe_experts(bank.experts, x, i32.long(), f32),
                 lambda: w2.moe_experts(bank.experts, x, i32, i32), lambda: w2.moe_experts(bank.experts, x, i32, f32[:, :1]),
                 lambda: w2.moe_experts(bank.experts, x, i32, f32, base=r), lambda: w2.moe_experts(bank.experts, x, i32, f32, out=x[:2])]:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(w2.W2Error):
        w2.moe_experts(bank.experts, x, i32, f32, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
