"""The operators between the projections against their definitions in 64 bits, and their refusals.

Bounds, with u = 2^-8 the relative error of one rounding to bf16 (8 significant bits) and e = 2^-24 that of fp32:
* rotation: |y| u for the rounding, and 2^-16 of the terms' magnitude for sine, cosine, norm and products (about ten fp32
  operations and a sine that is good to 2^-20);
* adapters: |y| u, and 2^-13 of the terms' magnitude: factors in two bf16 parts leave 2^-16 each, fp32 sums over K <= 2^14
  terms in ranges leave less than 2^-14 of the sum of magnitudes;
* attention: |y| u, and 2 u of sum p |v| for weights that are rounded to bf16 before they meet V (u for the weight, and the
  same again for a sum of weights that is not rounded); lse: (D + 8) e of the largest sum of |q||k| scale, and 2^-18.
"""
import ctypes
import math

import numpy as np
import pytest

from oracle import block_oracle as want

torch = pytest.importorskip("torch")
U = 2.0 ** -8


@pytest.fixture(scope="module")
def w2():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_06753_amd import binding
    return binding


def f64(t):
    return t.detach().double().cpu().numpy()


def near(got, ref, tol, what):
    got = f64(got) if torch.is_tensor(got) else got
    assert np.isfinite(got).all(), f"{what}: {np.count_nonzero(~np.isfinite(got))} outputs are not finite"
    off = np.abs(got - ref) - tol
    assert (off <= 0).all(), f"{what}: {np.count_nonzero(off > 0)} of {off.size} off, worst by {off.max():.3g} over its bound"


def normal(seed, *shape, dtype=torch.bfloat16, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


# ------------------------------------------------------------------ adapters
def lora_case(w2, M, K, parts, R, n, gated=False, act=0, xdt=torch.bfloat16, ranks=None, none=False, with_base=True,
              pad=0, seed=0, scales=True, in_place=False):
    N = sum(parts)
    P = 2 if gated else len(parts)
    rng = np.random.default_rng(seed)
    X = normal(seed + 1, M, K + pad, dtype=xdt)[:, :K]
    A = normal(seed + 2, n, P * R, K, std=K ** -0.5)
    B = normal(seed + 3, n, N, R, std=R ** -0.5)
    base = normal(seed + 4, M, N + pad)[:, :N] if with_base else None
    ad = rng.integers(-1 if none else 0, n, M).astype(np.int32)
    rank = None if ranks is None else torch.tensor([ranks[i % len(ranks)] for i in range(n)], dtype=torch.int32, device="cuda")
    scale = torch.tensor(rng.uniform(0.25, 2.0, n), dtype=torch.float32, device="cuda") if scales else None
    if rank is not None:                                      # what lies past an adapter's rank is not its own
        for i in range(n):
            r = min(max(int(rank[i]), 0), R)
            B[i, :, r:] = float("nan")
            for p in range(P):
                A[i, p * R + r:(p + 1) * R] = float("nan")
    lora = w2.Lora(A, B, rank=rank, scale=scale, parts=None if gated else parts, gated=gated)
    part = np.arange(N) // 16 % 2 if gated else np.repeat(np.arange(P), parts)
    ref, mag = want.lora(f64(X), np.nan_to_num(f64(A)), np.nan_to_num(f64(B)), ad, None if base is None else f64(base),
                         None if rank is None else rank.tolist(), None if scale is None else scale.tolist(), part, act)
    ws = torch.full((w2.lora_workspace_size(lora, M),), 0xff, dtype=torch.uint8, device="cuda")    # NaN to begin with
    out = base if in_place else torch.full((M, ref.shape[1] + pad), 3.0, dtype=torch.bfloat16, device="cuda")[:, :ref.shape[1]]
    Y = w2.lora_add(lora, X, torch.tensor(ad, device="cuda"), base, act=act, out=out, workspace=ws)
    assert Y is out
    near(Y, ref, U * np.abs(ref) + 2.0 ** -13 * mag, f"lora M={M} K={K} parts={parts} R={R} n={n}")
    if pad and not in_place:
        assert (out._base[:, ref.shape[1]:] == 3.0).all(), "columns past the row's end were written"
    return lora


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("xdt", [torch.bfloat16, torch.float32])
def test_lora_row_counts(w2, M, xdt):
    lora_case(w2, M, 512, [320, 80, 48], 16, 5, xdt=xdt, none=True, seed=M)


@pytest.mark.gpu
@pytest.mark.parametrize("R", [8, 16, 24, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("M", [1, 9, 70])
def test_lora_ranks(w2, R, M):
    lora_case(w2, M, 768, [208], R, 3, seed=R + M)
    lora_case(w2, M, 256, [64, 32, 16, 40], R, 4, ranks=[R, 1, 0, R - 3, -2, R + 9], seed=R + M + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("K,N", [(256, 8), (256, 24), (1280, 264), (4096, 128), (14336, 72), (17408, 16)])
@pytest.mark.parametrize("xdt", [torch.bfloat16, torch.float32])
def test_lora_shapes(w2, K, N, xdt):
    for M in (1, 20):
        lora_case(w2, M, K, [N], 16, 2, xdt=xdt, seed=K + N + M)


@pytest.mark.gpu
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M", [1, 37, 257])
def test_lora_activations_gated_strides(w2, act, gated, M):
    lora_case(w2, M, 512, [352], 32, 6, gated=gated, act=act, pad=24, none=True, ranks=[32, 7, 16], seed=act + M)
    lora_case(w2, M, 512, [352], 8, 1, gated=gated, act=act, with_base=False, scales=False, seed=act + M + 5)


@pytest.mark.gpu
@pytest.mark.parametrize("xdt", [torch.bfloat16, torch.float32])
def test_lora_many_rows_of_wide_factors(w2, xdt):
    # more rows of A than one workgroup takes, the last of them few; K in one to eight parts, of few and of many stages
    lora_case(w2, 400, 512, [160, 80, 48], 24, 3, xdt=xdt, none=True, seed=1)
    lora_case(w2, 330, 1280, [64, 32], 40, 2, xdt=xdt, ranks=[40, 9], seed=2)
    lora_case(w2, 150, 4352, [48], 128, 2, xdt=xdt, seed=3)
    lora_case(w2, 500, 768, [96], 128, 90, xdt=xdt, ranks=[128, 60, 0], none=True, seed=4)


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
def test_lora_many_rows_and_columns(w2, gated):
    # several steps of columns a workgroup, the last ones past the end, and windows of several adapters
    lora_case(w2, 900, 256, [4096 + 264 - 8 * gated], 8, 40, gated=gated, act=2 * gated, none=True, seed=5)
    lora_case(w2, 700, 256, [6016], 64, 2, gated=gated, act=2 * gated, pad=8, seed=6)
    lora_case(w2, 1100, 512, [2496], 128, 3, gated=gated, act=1, ranks=[128, 8, 33], seed=7)


@pytest.mark.gpu
def test_lora_in_place_all_none_and_many_adapters(w2):
    lora_case(w2, 50, 512, [96], 16, 3, in_place=True)
    lora_case(w2, 40, 512, [96], 16, 64, none=True)
    lora_case(w2, 200, 256, [96], 8, 150)
    X, A, B = normal(1, 5, 256), normal(2, 2, 8, 256), normal(3, 2, 32, 8)
    A[:] = float("nan")                                       # rows without an adapter do not meet one
    base = normal(4, 5, 32)
    ad = torch.tensor([-1, 2, 1 << 30, -(1 << 31), -7], dtype=torch.int32, device="cuda")
    Y = w2.lora_add(w2.Lora(A, B), X, ad, base)
    assert torch.equal(Y, base)


@pytest.mark.gpu
def test_lora_rows_do_not_depend_on_their_company(w2):
    # a row's result by itself and among others, in another order
    M, K, N, R, n = 48, 1024, 160, 16, 7
    X, base = normal(1, M, K), normal(2, M, N)
    lora = w2.Lora(normal(3, n, R, K, std=0.03), normal(4, n, N, R))
    ad = torch.tensor(np.random.default_rng(0).integers(-1, n, M).astype(np.int32), device="cuda")
    Y = w2.lora_add(lora, X, ad, base)
    perm = torch.randperm(M, generator=torch.Generator().manual_seed(1)).cuda()
    Z = w2.lora_add(lora, X[perm].contiguous(), ad[perm].contiguous(), base[perm].contiguous())
    assert torch.equal(Z, Y[perm])


# ------------------------------------------------------------------ norm, rotation, cache
def rope_case(w2, M, hq, hkv, D, rd, inter, norm, page=16, scaling=None, mscale=1.0, base=10000.0, top=4096, in_place=False,
              heads_first=False, seed=0, pad=0, holes=False, eps=1e-5, positions=None):
    rng = np.random.default_rng(seed)
    width = (hq + 2 * hkv) * D
    x = normal(seed + 1, M, width + pad)[:, :width]
    qw = (1 + normal(seed + 2, D, dtype=torch.float32, std=0.2)).bfloat16() if norm else None
    kw = (1 + normal(seed + 3, D, dtype=torch.float32, std=0.2)).bfloat16() if norm else None
    pos = rng.integers(0, top, M).astype(np.int32) if positions is None else np.asarray(positions, np.int32)
    pages = (M + page - 1) // page + 2
    slots = rng.permutation(pages * page)[:M].astype(np.int64)
    if holes:
        slots[::3] = -1
        slots[1] = pages * page
    if heads_first:
        k, v = (normal(seed + 4 + i, pages, hkv, page, D).transpose(1, 2) for i in (0, 1))
    else:
        k, v = (normal(seed + 4 + i, pages, page, hkv, D) for i in (0, 1))
    k0, v0 = f64(k).reshape(-1, hkv, D), f64(v).reshape(-1, hkv, D)
    x64 = f64(x).reshape(M, -1, D)
    rope = w2.Rope(rd, base=base, interleaved=inter, scaling=scaling, mscale=mscale) if rd else None
    theta = want.rope_frequencies(rd, base, scaling) if rd else None
    out = x[:, :hq * D].unflatten(1, (hq, D)) if in_place else None
    q = w2.qk_norm_rope(x, hq, rope, torch.tensor(pos, device="cuda"), w2.KVCache(k, v), torch.tensor(slots, device="cuda"),
                        q_weight=qw, k_weight=kw, eps=eps, out=out)
    what = f"rope M={M} heads={hq}/{hkv}/{D} rd={rd} inter={inter} norm={norm}"
    ref, mag = want.norm_rope(x64[:, :hq], f64(qw) if norm else None, eps, theta, inter, mscale, pos)
    near(q, ref, U * np.abs(ref) + 2.0 ** -16 * mag, what + " q")
    ref, mag = want.norm_rope(x64[:, hq:hq + hkv], f64(kw) if norm else None, eps, theta, inter, mscale, pos)
    live = (slots >= 0) & (slots < pages * page)
    tol = np.zeros_like(k0)
    k0[slots[live]], tol[slots[live]] = ref[live], (U * np.abs(ref) + 2.0 ** -16 * mag)[live]
    v0[slots[live]] = x64[live, hq + hkv:]
    near(f64(k).reshape(-1, hkv, D), k0, tol, what + " k")     # the other slots as they were
    assert np.array_equal(f64(v).reshape(-1, hkv, D), v0), what + " v"


@pytest.mark.gpu
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("hq,hkv,D,rd", [(32, 8, 128, 128), (4, 2, 64, 64), (3, 1, 128, 96), (8, 4, 256, 256), (5, 5, 80, 80),
                                         (15, 5, 96, 72), (21, 3, 80, 60), (2, 1, 8, 8), (2, 1, 8, 4), (6, 2, 24, 12),
                                         (1, 1, 256, 4), (9, 3, 256, 20), (64, 8, 128, 64), (2, 2, 40, 32), (7, 1, 248, 248)])
def test_rope_layouts(w2, inter, hq, hkv, D, rd):
    for M, norm in ((1, True), (3, False), (13, True)):
        rope_case(w2, M, hq, hkv, D, rd, inter, norm, seed=D + rd + M)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [1, 7, 16, 48, 64])
@pytest.mark.parametrize("heads_first", [False, True])
def test_rope_pages_and_holes(w2, page, heads_first):
    for M in (2, 37, 200):
        rope_case(w2, M, 6, 2, 64, 64, False, True, page=page, heads_first=heads_first, holes=True, seed=page + M, pad=40)


@pytest.mark.gpu
@pytest.mark.parametrize("scaling", [None, ("linear", 4.0), ("ntk", 8.0), ("bands", 8.0, 8192, 1.0, 4.0), ("bands", 32.0, 4096, 1.0, 32.0)])
def test_rope_scaled_and_far_positions(w2, scaling):
    # the angle is as exact at the last position as at the first
    far = [0, 1, 4095, 131071, 1000003, (1 << 24) + 1, (1 << 31) - 1]
    for inter in (False, True):
        rope_case(w2, len(far), 4, 2, 128, 128, inter, True, scaling=scaling, mscale=1.25, base=500000.0, positions=far)


@pytest.mark.gpu
def test_rope_in_place_no_rotation_no_slots(w2):
    rope_case(w2, 9, 4, 2, 64, 64, False, True, in_place=True)
    rope_case(w2, 9, 4, 2, 64, 32, True, False, in_place=True)
    rope_case(w2, 9, 4, 2, 96, 0, False, True)
    M, D = 5, 64
    x = normal(1, M, 6 * D)
    k, v = (torch.zeros(2, 4, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = w2.qk_norm_rope(x, 2, None, None, w2.KVCache(k, v))     # neither norm nor rotation: a copy to slots 0..M-1
    x = x.view(M, 6, D)
    assert torch.equal(q, x[:, :2]) and torch.equal(k.view(8, 2, D)[:M], x[:, 2:4]) and torch.equal(v.view(8, 2, D)[:M], x[:, 4:])
    assert not k.view(8, 2, D)[M:].any()


@pytest.mark.gpu
def test_rope_many_rows(w2):
    rope_case(w2, 1031, 10, 2, 128, 128, False, True, page=32, top=131072)


@pytest.mark.gpu
def test_rope_extreme_rows(w2):
    # a row of zeros, a large one and a tiny one: the norm's sum stays finite, eps holds up the zero row
    M, D = 4, 128
    x = normal(1, M, 3 * D)
    x[0] = 0
    x[1] *= 1e15
    x[2] *= 1e-15
    k, v = (torch.zeros(1, 4, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    q = w2.qk_norm_rope(x, 1, w2.Rope(D), torch.arange(4, dtype=torch.int32, device="cuda"), w2.KVCache(k, v), q_weight=w,
                        k_weight=w, eps=1e-6)
    ref, mag = want.norm_rope(f64(x)[:, None, :D], np.ones(D), 1e-6, want.rope_frequencies(D, 10000.0), False, 1.0, range(4))
    near(q, ref, U * np.abs(ref) + 2.0 ** -16 * mag, "extreme rows")


def test_rope_phases_on_host():
    from paper_2508_06753_amd import binding as w2
    for rd, base, scaling in [(128, 10000.0, None), (64, 500000.0, ("linear", 4.0)), (96, 1e6, ("ntk", 2.0)),
                              (128, 500000.0, ("bands", 8.0, 8192, 1.0, 4.0)), (4, 1.0, None)]:
        got = w2.rope_phases(rd, base, scaling).numpy().view(np.uint64)
        ref = want.rope_frequencies(rd, base, scaling) / (2 * math.pi) * 2.0 ** 64
        assert np.all(np.abs(got.astype(np.float64) - ref) <= 2.0 ** -46 * 2.0 ** 64)
    assert w2.rope_phases(8, 10000.0)[0] == int(2.0 ** 64 / (2 * math.pi))
    for bad in [dict(rotary_dim=6), dict(rotary_dim=0), dict(rotary_dim=260), dict(rotary_dim=8, base=0.5),
                dict(rotary_dim=8, scaling=("linear", 0.5)), dict(rotary_dim=8, scaling=("bands", 2.0, 0, 1.0, 2.0)),
                dict(rotary_dim=8, scaling=("bands", 2.0, 100, 2.0, 2.0)), dict(rotary_dim=8, base=float("nan"))]:
        with pytest.raises(w2.W2Error):
            w2.rope_phases(**bad)
    with pytest.raises(ValueError):
        w2.rope_phases(8, scaling=("linear",))


# ------------------------------------------------------------------ attention
def tree_masks(T, rng):
    words = (T + 63) // 64
    bits = []
    for i in range(T):
        parent = int(rng.integers(max(-1, i - 5), i)) if i else -1
        bits.append((bits[parent] if parent >= 0 else 0) | 1 << i)
    return np.array([[b >> (64 * w) & (1 << 64) - 1 for w in range(words)] for b in bits], np.uint64).reshape(T, words)


def tree_case(w2, requests, hq, hkv, D, page=16, masked=True, seed=0, scale=None, split=True, heads_first=False, pad=0,
              absent=False, masks=None, q_std=1.5, total=True, spoil=True, slack=0, lse=True):
    """requests: [(keys, drafted tokens)]"""
    rng = np.random.default_rng(seed)
    R, M = len(requests), sum(t for _, t in requests)
    need = [(n + page - 1) // page for n, _ in requests]
    pages = sum(need) + 3
    order = rng.permutation(pages).astype(np.int32)
    cols = max(need + [1]) + 1
    table = np.full((R, cols), -1, np.int32)
    at = 0
    for r, c in enumerate(need):
        table[r, :c] = order[at:at + c]
        at += c
    shape = (pages, hkv, page, D) if heads_first else (pages, page, hkv, D)
    k, v = normal(seed + 1, *shape), normal(seed + 2, *shape)
    if heads_first:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    kf, vf = f64(k).reshape(-1, hkv, D), f64(v).reshape(-1, hkv, D)
    q = normal(seed + 3, M, hq * D + pad, std=q_std)[:, :hq * D].unflatten(1, (hq, D))
    words = max((t + 63) // 64 for _, t in requests)
    mask = np.zeros((M, max(1, words)), np.uint64)
    refs = ([], [], [])
    big, used, row = 0.0, np.zeros(pages * page, bool), 0
    scale_ = D ** -0.5 if scale is None else scale
    for r, (n, t) in enumerate(requests):
        if absent and need[r] > 1:
            table[r, rng.integers(0, need[r])] = [-1, pages, 1 << 30][r % 3]
        own = tree_masks(t, rng) if masks is None else masks[r]
        if t:
            mask[row:row + t, :own.shape[1]] = own
        c = np.arange(n)
        p = table[r, c // page]
        there = (p >= 0) & (p < pages)
        slot = np.where(there, p, 0).astype(np.int64) * page + c % page
        used[slot[there]] = True
        kk, vv = kf[slot].copy(), vf[slot]
        kk[~there] = np.nan
        o, l, mg, b = want.attention(f64(q)[row:row + t], kk, vv, t, mask[row:row + t] if masked else None, scale_)
        for dst, x in zip(refs, (o, l, mg)):
            dst.append(x)
        big = max(big, b)
        row += t
    if spoil:                                                  # what no request owns may hold anything
        kv = k.reshape(-1, hkv, D) if not heads_first else None
        bad = torch.tensor(~used, device="cuda")
        for tns, val in ((k, float("nan")), (v, float("inf"))):
            tns[bad.view(pages, page)] = val
        del kv
    cache = w2.KVCache(k, v)
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    starts = np.concatenate([[0], np.cumsum([t for _, t in requests])])
    most_t, most_n = max(t for _, t in requests) + slack, max(n for n, _ in requests) + 37 * slack
    total_len = sum(n for n, _ in requests) if total else 0
    ws = None
    if split:
        ws = torch.full((max(16, w2.tree_attention_workspace_size(R, M, hq, cache, most_t, most_n, total_len)),), 0xff,
                        dtype=torch.uint8, device="cuda")
    out = torch.full((M, hq * D + pad), 7.0, dtype=torch.bfloat16, device="cuda")[:, :hq * D].unflatten(1, (hq, D))
    L = torch.full((M, hq), 9.0, device="cuda") if lse else None
    w2.tree_attention(q, cache, i32(table), i32(starts), i32([n for n, _ in requests]), most_t, most_n,
                      mask=torch.tensor(mask.view(np.int64), device="cuda") if masked else None, scale=scale,
                      total_len=total_len, out=out, lse=L, workspace=ws)
    what = f"tree {requests} heads={hq}/{hkv}/{D} page={page} masked={masked}"
    ref, ref_l, mag = (np.concatenate(x) for x in refs)
    near(out, ref, U * np.abs(ref) + 2 * U * mag, what)
    if lse:
        got = f64(L)
        empty = np.isinf(ref_l)
        assert np.array_equal(np.isneginf(got), empty), what + ": lse of rows that see nothing"
        near(got[~empty], ref_l[~empty], (D + 8) * 2.0 ** -24 * big + 2.0 ** -18, what + " lse")
    if pad:
        assert (out._base[:, hq * D:] == 7.0).all()
    return out, L


HEADS = [(32, 8, 128), (4, 4, 64), (8, 4, 256), (6, 1, 96), (21, 3, 80), (16, 1, 128), (2, 2, 8), (5, 1, 40), (3, 1, 248)]


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D", HEADS)
@pytest.mark.parametrize("split", [False, True])
def test_tree_heads(w2, hq, hkv, D, split):
    tree_case(w2, [(300, 1)], hq, hkv, D, split=split, masked=False, seed=D)
    tree_case(w2, [(77, 7), (1, 1), (260, 12)], hq, hkv, D, split=split, seed=D + 1)
    tree_case(w2, [(140, 70), (33, 33)], hq, hkv, D, split=split, masked=False, seed=D + 2)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1025])
def test_tree_key_counts(w2, n):
    for t in {1, min(n, 5)}:
        tree_case(w2, [(n, t)], 8, 2, 64, seed=n + t)
        tree_case(w2, [(n, t)], 4, 1, 128, masked=False, page=32, seed=n + t)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 33, 63, 64, 65, 100, 130, 200])
def test_tree_row_counts(w2, t):
    # masks of up to four words
    tree_case(w2, [(t + 90, t)], 8, 2, 64, seed=t)
    tree_case(w2, [(t, t), (t + 1, 1)], 4, 4, 128, seed=t + 1)
    tree_case(w2, [(t + 9, t)], 3, 1, 128, masked=False, seed=t + 2)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [1, 5, 8, 16, 24, 64, 100, 256, 1000])
@pytest.mark.parametrize("heads_first", [False, True])
def test_tree_pages(w2, page, heads_first):
    tree_case(w2, [(333, 9), (64, 3), (5, 5)], 8, 2, 64, page=page, heads_first=heads_first, seed=page)
    tree_case(w2, [(210, 40), (64, 3)], 8, 2, 128, page=page, heads_first=heads_first, seed=page, absent=True)


@pytest.mark.gpu
@pytest.mark.parametrize("split", [False, True])
def test_tree_rows_that_see_nothing(w2, split):
    nothing = np.zeros((6, 1), np.uint64)
    some = np.array([[0], [1], [0], [8], [63], [0]], np.uint64)
    for hq, hkv, D in ((4, 2, 64), (8, 1, 128)):
        tree_case(w2, [(6, 6), (6, 6), (200, 6)], hq, hkv, D, masks=[nothing, some, nothing], split=split)
    # requests without rows, without keys, with more rows than keys
    tree_case(w2, [(40, 0), (0, 3), (2, 5), (90, 2)], 4, 2, 64, split=split)
    tree_case(w2, [(40, 0), (0, 3), (2, 5), (90, 2)], 4, 2, 64, split=split, masked=False)


@pytest.mark.gpu
def test_tree_ragged_batches_strides_scales(w2):
    reqs = [(2000, 1), (3, 1), (900, 1), (64, 1), (1, 1), (1500, 1)]
    tree_case(w2, reqs, 16, 4, 128, masked=False, pad=72)
    tree_case(w2, reqs, 16, 4, 64, masked=False, total=False, slack=3, lse=False)
    tree_case(w2, [(700, 20), (1300, 64), (65, 2)], 16, 4, 128, scale=0.5, slack=2)
    tree_case(w2, [(700, 20)], 8, 2, 64, scale=-0.125)
    tree_case(w2, [(700, 20)], 8, 2, 64, scale=0.0)
    tree_case(w2, [(900, 3)], 8, 2, 64, q_std=60.0)              # one key takes nearly all the weight
    tree_case(w2, [(n % 97 + 1, 1) for n in range(0, 2000, 17)], 4, 2, 64, masked=False)


@pytest.mark.gpu
def test_tree_long(w2):
    tree_case(w2, [(20011, 2)], 8, 2, 128, page=64, seed=5)
    tree_case(w2, [(9000, 33), (4001, 1)], 8, 2, 64, page=32, seed=6)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D", [(4, 1, 128), (8, 2, 64), (8, 4, 256), (5, 1, 128), (16, 2, 128), (12, 2, 96)])
def test_tree_many_rows_over_long_contexts(w2, hq, hkv, D):
    # two and four waves, chunks with a middle that nothing is checked in, and the same with pages that are not there
    for t in (12, 40):
        for absent in (False, True):
            tree_case(w2, [(1500, t), (333, 3)], hq, hkv, D, page=32, absent=absent, seed=t + D)
            tree_case(w2, [(1100, t)], hq, hkv, D, page=16, absent=absent, masked=False, split=False, seed=t + D + 1)
        tree_case(w2, [(900, t)], hq, hkv, D, page=40, seed=t + D + 2)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D", [(21, 3, 80), (5, 1, 40), (15, 5, 96), (6, 2, 72), (6, 2, 248)])
def test_tree_padded_heads_over_long_contexts(w2, hq, hkv, D):
    # heads shorter than the kernel's rows, in the middle of a chunk; what lies behind a head belongs to the next one
    for t, split in ((13, True), (13, False), (50, True), (50, False)):
        tree_case(w2, [(1200, t), (600, t - 5)], hq, hkv, D, page=48, split=split, seed=t + D)
        tree_case(w2, [(1000, t)], hq, hkv, D, page=16, masked=False, split=split, heads_first=True, seed=t + D + 1)


@pytest.mark.gpu
def test_tree_many_units_and_chunks_of_one_length(w2):
    # more units than run at once, and few over many keys: chunks by either rule
    tree_case(w2, [(300 + 7 * i, 40) for i in range(20)], 16, 4, 128, page=32, seed=1)
    tree_case(w2, [(260 + 9 * i, 70) for i in range(9)], 32, 16, 64, masked=False, seed=2)
    tree_case(w2, [(7001, 20)], 8, 2, 128, page=16, seed=3)
    tree_case(w2, [(7001, 20), (40, 20)], 8, 2, 128, page=16, total=False, slack=1, seed=4)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [640, 700, 768, 769, 1000, 1024, 1025])
def test_tree_short_requests_in_one_launch(w2, n):
    tree_case(w2, [(n, 1)], 8, 2, 128, masked=False, seed=n)
    tree_case(w2, [(n, 3), (n - 600, 1)], 8, 4, 64, seed=n + 1)
    tree_case(w2, [(n - i, 1) for i in range(16)], 8, 8, 64, masked=False, seed=n + 2)


@pytest.mark.gpu
def test_tree_one_token_is_row_of_a_chunk(w2):
    # the last row of a causal chunk is the single token of the same request
    out, lse = tree_case(w2, [(500, 50)], 8, 2, 128, masked=False, seed=3)
    assert out.shape[0] == 50 and lse.shape == (50, 8)


@pytest.mark.gpu
def test_tree_far_pages(w2):
    # a cache whose pages lie past 2^31 elements
    D, page = 128, 16
    pages = (1 << 31) // (page * 4 * D) + 40
    k = torch.empty(pages, page, 4, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty(pages, page, 4, D, dtype=torch.bfloat16, device="cuda")
    n = 200
    ids = np.array([pages - 1 - 3 * i for i in range((n + page - 1) // page)], np.int32)
    x = normal(1, n, 12 * D)
    slots = np.repeat(ids.astype(np.int64), page)[:n] * page + np.arange(n) % page
    cache = w2.KVCache(k, v)
    q = w2.qk_norm_rope(x, 4, w2.Rope(D), torch.arange(n, dtype=torch.int32, device="cuda"), cache, torch.tensor(slots, device="cuda"))
    i32 = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
    out = w2.tree_attention(q[-3:], cache, i32(ids[None]), i32([0, 3]), i32([n]), 3, n)
    kk, _ = want.norm_rope(f64(x).reshape(n, 12, D)[:, 4:8], None, 0.0, want.rope_frequencies(D, 10000.0), False, 1.0, range(n))
    kk = f64(torch.tensor(kk).bfloat16())
    ref, _, mag, _ = want.attention(f64(q[-3:]), kk, f64(x).reshape(n, 12, D)[:, 8:], 3, None, D ** -0.5)
    # a key rounded the other way moves its weight by up to its score's change
    near(out, ref, U * np.abs(ref) + 4 * U * mag, "far pages")


# ------------------------------------------------------------------ streams and graphs
@pytest.mark.gpu
def test_block_ops_on_a_stream_and_in_a_graph(w2):
    M, D, hq, hkv, K, n = 6, 64, 4, 2, 256, 150
    width = (hq + 2 * hkv) * D
    x, base = normal(1, M, K), normal(2, M, width)
    lora = w2.Lora(normal(3, 3, 3 * 8, K, std=0.06), normal(4, 3, width, 8), parts=[hq * D, hkv * D, hkv * D])
    i32 = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
    ad, pos, start, lens = i32([0, 2, 1, -1, 2, 2]), i32([100, 101, 102, 60, 61, 61]), i32([0, 3, 6]), i32([103, 62])
    k, v = normal(5, 20, 16, hkv, D), normal(6, 20, 16, hkv, D)
    table = i32(np.arange(14).reshape(2, 7))
    slots = torch.tensor([6 * 16 + 4, 6 * 16 + 5, 6 * 16 + 6, 10 * 16 + 11, 10 * 16 + 12, 10 * 16 + 13], device="cuda")
    cache, rope = w2.KVCache(k, v), w2.Rope(D)
    ws = torch.empty(w2.lora_workspace_size(lora, M), dtype=torch.uint8, device="cuda")
    wt = torch.empty(max(16, w2.tree_attention_workspace_size(2, M, hq, cache, 3, 103)), dtype=torch.uint8, device="cuda")
    y, q, o = torch.empty_like(base), torch.empty(M, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(M, hq, D, dtype=torch.bfloat16, device="cuda")

    def step():
        w2.lora_add(lora, x, ad, base, out=y, workspace=ws)
        w2.qk_norm_rope(y, hq, rope, pos, cache, slots, out=q)
        w2.tree_attention(q, cache, table, start, lens, 3, 103, out=o, workspace=wt)

    step()
    torch.cuda.synchronize()
    eager = o.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o.zero_()
        step()
    side.synchronize()
    assert torch.equal(o, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        fresh = normal(10 + i, M, K)
        x.copy_(fresh)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, o), f"replay {i}"


# ------------------------------------------------------------------ refusals (no device is touched)
def test_refusals_of_the_c_entries():
    from paper_2508_06753_amd import binding as w2
    lib = w2.raw()
    P = 4096                                                   # an aligned address that is never followed
    out = ctypes.c_size_t(0)

    def lora(**kw):
        f = dict(A=P, B=P, rank=None, scale=None, a_stride=256 * 16, b_stride=64 * 16, n_adapters=2, max_rank=16, n_parts=2, gated=0)
        ends = kw.pop("ends", (32, 64, 0, 0))
        f.update(kw)
        return w2._LoraStruct(part_end=(ctypes.c_int64 * 4)(*ends), **f)

    def add(l=None, K=256, N=64, X=P, dt=1, ldx=256, M=3, ad=P, base=P, ldb=64, Y=2 * P, ldy=64, act=0, ws=P, wb=1 << 20):
        return lib.w2_lora_add(ctypes.byref(l or lora()), K, N, X, dt, ldx, M, ad, base, ldb, Y, ldy, act, ws, wb, None)

    INV, SHAPE, ALIGN, SMALL = w2.ERR_INVALID_ARG, w2.ERR_UNSUPPORTED_SHAPE, w2.ERR_MISALIGNED, w2.ERR_BUFFER_TOO_SMALL
    assert add(M=0, X=None, ad=None, Y=None, ws=None) == 0
    for want_rc, kw in [(INV, dict(X=None)), (INV, dict(ad=None)), (INV, dict(Y=None)), (INV, dict(l=lora(A=None))), (INV, dict(M=-1)),
                        (INV, dict(dt=5)), (INV, dict(act=3)), (INV, dict(l=lora(n_parts=5))), (INV, dict(l=lora(n_parts=0))),
                        (INV, dict(l=lora(ends=(32, 48, 0, 0)))), (INV, dict(l=lora(ends=(64, 64, 0, 0)))), (INV, dict(l=lora(n_adapters=0))),
                        (SHAPE, dict(l=lora(ends=(24, 64, 0, 0)))), (SHAPE, dict(K=255)), (SHAPE, dict(N=60)), (SHAPE, dict(l=lora(max_rank=12))),
                        (SHAPE, dict(l=lora(max_rank=136))), (SHAPE, dict(N=40, act=2, l=lora(n_parts=1, ends=(40, 0, 0, 0)))),
                        (SHAPE, dict(N=40, l=lora(gated=1))), (SHAPE, dict(M=1 << 25)),
                        (ALIGN, dict(X=P + 8)), (ALIGN, dict(Y=P + 2)), (ALIGN, dict(ldx=252)), (ALIGN, dict(ldy=60)), (ALIGN, dict(ldb=8)),
                        (ALIGN, dict(l=lora(a_stride=4))), (ALIGN, dict(l=lora(B=P + 4))), (ALIGN, dict(ws=P + 4)),
                        (SMALL, dict(wb=8)), (SMALL, dict(ws=None)), (INV, dict(act=2, Y=P, ldy=64))]:
        assert add(**kw) == want_rc, kw
        assert lib.w2_last_error() != b""
    assert lib.w2_lora_add(None, 256, 64, P, 1, 256, 1, P, P, 64, P, 64, 0, P, 1 << 20, None) == INV
    assert lib.w2_lora_workspace_size(ctypes.byref(lora()), 3, 256, 64, None) == INV
    assert lib.w2_lora_workspace_size(ctypes.byref(lora()), 3, 256, 64, ctypes.byref(out)) == 0 and out.value >= 3 * 32 * 4

    def cache(**kw):
        f = dict(k=P, v=P, n_pages=4, page_size=16, k_page_stride=2048, k_slot_stride=128, k_head_stride=64, v_page_stride=2048,
                 v_slot_stride=128, v_head_stride=64, n_heads=2, head_dim=64)
        f.update(kw)
        return w2._CacheStruct(**f)

    bad_caches = [(INV, cache(k=None)), (INV, cache(n_pages=0)), (INV, cache(page_size=0)), (INV, cache(n_heads=0)), (SHAPE, cache(head_dim=60)),
                  (SHAPE, cache(head_dim=264)), (SHAPE, cache(n_pages=1 << 30, page_size=4)), (ALIGN, cache(v=P + 8)),
                  (ALIGN, cache(k_slot_stride=4)), (ALIGN, cache(v_head_stride=-8)), (SHAPE, cache(n_pages=1 << 62, page_size=4))]

    def rope(c=None, r=w2._RopeStruct(P, 64, 0, 1.0), x=P, ldx=512, M=2, nq=4, qw=P, kw=P, eps=1e-6, pos=P, q=2 * P, ldq=256, slots=P):
        return lib.w2_qk_norm_rope(x, ldx, M, nq, qw, kw, eps, ctypes.byref(r) if r else None, pos, q, ldq, ctypes.byref(c or cache()), slots, None)

    assert rope(M=0, x=None, q=None, pos=None, slots=None) == 0
    for rc, c in bad_caches:
        assert rope(c=c) == rc
    for rc, kw in [(INV, dict(x=None)), (INV, dict(q=None)), (INV, dict(pos=None)), (INV, dict(M=-1)), (INV, dict(nq=0)), (INV, dict(eps=-1.0)),
                   (INV, dict(r=w2._RopeStruct(None, 64, 0, 1.0))), (SHAPE, dict(r=w2._RopeStruct(P, 66, 0, 1.0))),
                   (SHAPE, dict(r=w2._RopeStruct(P, 6, 0, 1.0))), (SHAPE, dict(r=w2._RopeStruct(P, 68, 0, 1.0))), (ALIGN, dict(ldx=504)),
                   (ALIGN, dict(ldq=260)), (ALIGN, dict(x=P + 2)), (ALIGN, dict(kw=P + 2)), (ALIGN, dict(r=w2._RopeStruct(P + 4, 64, 0, 1.0))),
                   (INV, dict(q=P, ldq=520)), (SMALL, dict(slots=None, M=65))]:
        assert rope(**kw) == rc, kw
    assert lib.w2_qk_norm_rope(P, 512, 1, 4, None, None, 0.0, None, None, P, 512, None, None, None) == INV

    def tree(c=None, q=P, ldq=256, M=3, nq=4, table=P, cols=4, ldt=4, start=P, lens=P, R=2, rows=2, length=60, total=0, mask=P, words=1,
             scale=0.125, o=P, ldo=256, lse=P, ws=None, wb=0):
        return lib.w2_tree_attention(q, ldq, M, nq, ctypes.byref(c or cache()), table, cols, ldt, start, lens, R, rows, length, total, mask,
                                     words, scale, o, ldo, lse, ws, wb, None)

    assert tree(M=0, q=None, o=None) == 0 and tree(R=0, start=None) == 0 and tree(rows=0) == 0
    for rc, c in bad_caches:
        assert tree(c=c) == rc
    for rc, kw in [(INV, dict(q=None)), (INV, dict(o=None)), (INV, dict(table=None)), (INV, dict(start=None)), (INV, dict(lens=None)),
                   (INV, dict(words=0)), (INV, dict(M=-1)), (INV, dict(R=-1)), (INV, dict(rows=-1)), (INV, dict(length=-1)), (INV, dict(total=-1)),
                   (INV, dict(ldt=3)), (INV, dict(cols=-1)), (INV, dict(scale=float("nan"))), (INV, dict(scale=float("inf"))), (INV, dict(nq=0)),
                   (SHAPE, dict(nq=5)), (SHAPE, dict(R=65536)), (SHAPE, dict(M=1 << 25)), (SHAPE, dict(length=1 << 31)), (SHAPE, dict(nq=2048)),
                   (ALIGN, dict(q=P + 8)), (ALIGN, dict(o=P + 2)), (ALIGN, dict(ldq=252)), (ALIGN, dict(ldo=260)), (ALIGN, dict(mask=P + 4)),
                   (ALIGN, dict(lse=P + 2)), (ALIGN, dict(ws=P + 8, wb=64))]:
        assert tree(**kw) == rc, kw
    size = lib.w2_tree_attention_workspace_size
    assert size(2, 3, 4, 2, 64, 2, 60, 0, None) == INV and size(2, 3, 4, 3, 64, 2, 60, 0, ctypes.byref(out)) == SHAPE
    assert size(2, 3, 4, 2, 60, 2, 60, 0, ctypes.byref(out)) == SHAPE and size(-2, 3, 4, 2, 64, 2, 60, 0, ctypes.byref(out)) == INV
    for big in (1 << 24, 65535):
        assert size(65535, big, 1024, 1, 256, big, (1 << 31) - 1, 0, ctypes.byref(out)) == 0


def test_refusals_of_the_binding():
    from paper_2508_06753_amd import binding as w2
    t = torch.zeros(2, 4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        w2.KVCache(t, t)                                       # host tensors
    with pytest.raises(ValueError):
        w2.Lora(torch.zeros(1, 8, 256, dtype=torch.bfloat16), torch.zeros(1, 16, 8, dtype=torch.bfloat16))


@pytest.mark.gpu
def test_refusals_of_the_binding_on_device_tensors(w2):
    A, B = normal(1, 2, 16, 256), normal(2, 2, 64, 16)
    lora = w2.Lora(A, B)
    X, base, ad = normal(3, 3, 256), normal(4, 3, 64), torch.zeros(3, dtype=torch.int32, device="cuda")
    for call in [lambda: w2.Lora(A.float(), B), lambda: w2.Lora(A, B, parts=[32, 16]), lambda: w2.Lora(A, B, gated=True),
                 lambda: w2.Lora(A, B, gated=True, parts=[64]), lambda: w2.Lora(A[:1], B), lambda: w2.Lora(A, B, rank=ad),
                 lambda: w2.lora_add(lora, X.half(), ad, base), lambda: w2.lora_add(lora, X[:, :128], ad, base),
                 lambda: w2.lora_add(lora, X, ad.long(), base), lambda: w2.lora_add(lora, X, ad[:2], base),
                 lambda: w2.lora_add(lora, X, ad, base[:, :32]), lambda: w2.lora_add(lora, X, ad, base, out=base[:, :32]),
                 lambda: w2.lora_add(lora, X, ad, base.float())]:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(w2.W2Error):
        w2.lora_add(lora, X, ad, base, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    k = normal(5, 4, 16, 2, 64)
    cache = w2.KVCache(k, k.clone())
    x, pos = normal(6, 3, 8 * 64), torch.zeros(3, dtype=torch.int32, device="cuda")
    q, one = normal(7, 3, 4, 64), torch.ones(1, dtype=torch.int32, device="cuda")
    table, start = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    for call in [lambda: w2.KVCache(k, k[:2]), lambda: w2.KVCache(k[0], k[0]), lambda: w2.KVCache(k.float(), k),
                 lambda: w2.qk_norm_rope(x, 5, None, None, cache), lambda: w2.qk_norm_rope(x, 4, None, pos.long(), cache),
                 lambda: w2.qk_norm_rope(x, 4, None, pos, cache, slots=pos), lambda: w2.qk_norm_rope(x, 4, None, pos, cache, out=q[:2]),
                 lambda: w2.qk_norm_rope(x, 4, None, pos, cache, q_weight=x[0]),
                 lambda: w2.tree_attention(q[..., :32], cache, table, start, one, 3, 16),
                 lambda: w2.tree_attention(q, cache, table, start[:1], one, 3, 16),
                 lambda: w2.tree_attention(q, cache, table.long(), start, one, 3, 16),
                 lambda: w2.tree_attention(q, cache, table, start, one, 3, 16, mask=start),
                 lambda: w2.tree_attention(q, cache, table, start, one, 3, 16, out=q[:, :2]),
                 lambda: w2.tree_attention(q, cache, table, start, one, 3, 16, lse=q[:, :, 0])]:
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------ the operators together
def block_and_cache(w2, adapters=True):
    from paper_2508_06753_amd import attention_block as ab, synth
    hidden, n_q, n_kv, D, G = 512, 4, 2, 64, 64
    width = (n_q + 2 * n_kv) * D

    def packed(K, N, seed):
        codes, scales = synth.make_weights(K, N, G, 0, seed=seed)
        return w2.prepack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales.view(np.int16)).cuda(), G)

    qkv = w2.Lora(normal(11, 2, 3 * 8, hidden, std=0.04), normal(12, 2, width, 8), parts=[n_q * D, n_kv * D, n_kv * D])
    o = w2.Lora(normal(13, 2, 8, n_q * D, std=0.06), normal(14, 2, hidden, 8))
    w = [(1 + normal(15 + i, D, dtype=torch.float32, std=0.2)).bfloat16() for i in (0, 1)]
    block = ab.AttentionBlock(packed(hidden, width, 1), packed(n_q * D, hidden, 2), hidden, n_q, n_kv, D, G, w2.Rope(D), *w,
                              qkv_lora=qkv if adapters else None, o_lora=o if adapters else None)
    k = normal(17, 24, 16, n_kv, D)
    return ab, block, w2.KVCache(k, torch.zeros_like(k))


@pytest.mark.gpu
def test_block_runs_prompts_trees_and_tokens(w2):
    """A step of the block against the operators' definitions on the projections that the library computes, and a drafted
    branch against the same tokens as a plain sequence."""
    ab, block, cache = block_and_cache(w2)
    table = torch.arange(20, dtype=torch.int32).flip(0).view(2, 10).contiguous().cuda()
    adapter, lens = [1, -1], [45, 70]
    D, n_q, n_kv = block.head_dim, block.n_q, block.n_kv
    history = [[], []]                                         # float64 keys and values of every committed token

    def check(batch, X, y, commit):
        M, starts = X.shape[0], batch.row_start.tolist()
        qkv = w2.matmul_a8_fused(block.wqkv, block.hidden, block.width, block.G, X,
                                 workspace=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"))
        ad = batch.adapter.cpu().numpy()
        part = np.repeat([0, 1, 2], [n_q * D, n_kv * D, n_kv * D])
        z, _ = want.lora(f64(X), f64(block.qkv_lora.A), f64(block.qkv_lora.B), ad, f64(qkv), part_of_column=part)
        z = f64(torch.tensor(z).bfloat16()).reshape(M, -1, D)
        pos, theta = batch.positions.tolist(), want.rope_frequencies(D, 10000.0)
        q, _ = want.norm_rope(z[:, :n_q], f64(block.q_weight), block.eps, theta, False, 1.0, pos)
        k, _ = want.norm_rope(z[:, n_q:n_q + n_kv], f64(block.k_weight), block.eps, theta, False, 1.0, pos)
        out = np.zeros((M, n_q, D))
        for r in range(2):
            rows = slice(starts[r], starts[r + 1])
            kk = np.stack([t[0] for t in history[r]] + list(k[rows]))
            vv = np.stack([t[1] for t in history[r]] + list(z[rows, n_q + n_kv:]))
            mask = None if batch.mask is None else batch.mask.cpu().numpy().view(np.uint64)[rows]
            out[rows] = want.attention(q[rows], kk, vv, starts[r + 1] - starts[r], mask, D ** -0.5)[0]
            if commit:
                history[r] += [(k[i], z[i, n_q + n_kv:]) for i in range(starts[r], starts[r + 1])]
        o = torch.tensor(out.reshape(M, -1)).bfloat16().cuda()
        base = w2.matmul_a8_fused(block.wo, n_q * D, block.hidden, block.G, o,
                                  workspace=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"))
        ref, _ = want.lora(f64(o), f64(block.o_lora.A), f64(block.o_lora.B), ad, f64(base))
        # a bf16 number rounded the other way somewhere moves the int8 codes of its row: compare the rows' norms of the difference
        off = np.linalg.norm(f64(y) - ref, axis=1) / np.linalg.norm(ref, axis=1)
        assert off.max() < 0.02, off

    def run(batch, seed, commit):
        X = normal(seed, batch.positions.shape[0], block.hidden, dtype=torch.float32)
        y = block.step(X, cache, batch)
        check(batch, X, y, commit)
        return X, y

    run(ab.causal_batch([0, 0], lens, table, 16, "cuda", adapter), 21, True)
    X, tree = run(ab.tree_batch(lens, [[-1, 0, 0, 1, 2], [-1, 0, 1]], table, 16, "cuda", adapter), 22, False)
    # the branch 0, 2, 4 of request 0, alone, as a plain continuation (request 1: all of its tree is one branch)
    pick = [0, 2, 4, 5, 6, 7]
    batch = ab.causal_batch(lens, [3, 3], table, 16, "cuda", adapter)
    line = block.step(X[pick].contiguous(), cache, batch)
    off = (line.float() - tree[pick].float()).norm(dim=1) / tree[pick].float().norm(dim=1)
    assert off.max().item() < 0.02, off


@pytest.mark.gpu
def test_block_without_adapters_and_main(w2, capsys):
    ab, block, cache = block_and_cache(w2, adapters=False)
    table = torch.arange(20, dtype=torch.int32).view(2, 10).contiguous().cuda()
    batch = ab.causal_batch([0, 0], [5, 1], table, 16, "cuda")
    y = block.step(normal(1, 6, block.hidden), cache, batch)
    assert y.shape == (6, block.hidden) and torch.isfinite(y).all()
    ab.main()
    said = capsys.readouterr().out
    assert said.count("finite True") == 3
