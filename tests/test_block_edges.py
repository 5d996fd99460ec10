"""The operators between the projections where numbers are not finite, lengths disagree and buffers are shared.

Bounds as in test_block_ops.py.  Where a number that is not finite reaches a result by the formula, the result's numbers that it
reaches are compared by kind (NaN, +infinity, -infinity), all others as usual.
"""
import ctypes

import numpy as np
import pytest

from oracle import block_oracle as want
from test_block_ops import U, block_and_cache, f64, near, normal, tree_masks

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def w2():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_06753_amd import binding
    return binding


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


# ------------------------------------------------------------------ the block's workspace
def test_a_step_keeps_no_memory(monkeypatch):
    """Every call of a step gets the caller's workspace, or one that is the step's own; the block holds none behind it."""
    from paper_2508_06753_amd import attention_block as ab
    given = []

    def call(shape):
        def run(*args, workspace=None, out=None, **kw):
            given.append(workspace)
            return torch.zeros(shape(*args)) if out is None else out
        return run

    hidden, n_q, n_kv, D = 512, 4, 2, 64
    width = (n_q + 2 * n_kv) * D
    sizes = dict(matmul=0)
    monkeypatch.setattr(ab.w2, "workspace_size", lambda *a: sizes["matmul"])
    monkeypatch.setattr(ab.w2, "tree_attention_workspace_size", lambda *a: 1000)
    monkeypatch.setattr(ab.w2, "lora_workspace_size", lambda *a: 300)
    monkeypatch.setattr(ab.w2, "matmul_a8_fused", call(lambda w, K, N, G, X: (X.shape[0], N)))
    monkeypatch.setattr(ab.w2, "lora_add", call(None))
    monkeypatch.setattr(ab.w2, "qk_norm_rope", lambda x, n, *a, **kw: torch.zeros(x.shape[0], n, D))
    monkeypatch.setattr(ab.w2, "tree_attention", call(lambda q, *a: q.shape))
    lora = object()
    block = ab.AttentionBlock(None, None, hidden, n_q, n_kv, D, 64, None, qkv_lora=lora, o_lora=lora)
    state = dict(vars(block))
    zeros = torch.zeros(2, dtype=torch.int32)
    batch = ab.Batch(zeros, zeros.long(), zeros.view(2, 1), torch.zeros(3, dtype=torch.int32), zeros, 1, 1, adapter=zeros)
    X = torch.zeros(2, hidden)
    assert block.workspace_size(2, batch, None) == 1000
    block.step(X, None, batch)
    first = list(given)
    assert len(first) == 5 and all(w is first[0] and w.numel() >= 1000 for w in first)
    sizes["matmul"] = 5000
    block.step(X, None, batch)
    assert len(given) == 10 and all(w is given[5] and w.numel() >= 5000 for w in given[5:])
    assert given[5].data_ptr() != first[0].data_ptr(), "two steps that have not run share memory"
    assert vars(block) == state, "the block holds what a step used"
    mine = torch.zeros(6000, dtype=torch.uint8)
    block.step(X, None, batch, workspace=mine)
    assert len(given) == 15 and all(w is mine for w in given[10:])
    with pytest.raises(ValueError):
        block.step(X, None, batch, workspace=mine[:4999])
    assert len(given) == 15


@pytest.mark.gpu
@pytest.mark.parametrize("own", [False, True])
def test_a_captured_step_outlives_larger_ones(w2, own):
    """A graph of a small step replayed behind a larger eager one: its result, and nothing of what was allocated since."""
    ab, block, cache = block_and_cache(w2)
    table = torch.arange(20, dtype=torch.int32).view(2, 10).contiguous().cuda()
    block.step(normal(1, 90, block.hidden, dtype=torch.float32), cache, ab.causal_batch([0, 0], [50, 40], table, 16, "cuda", [0, 1]))
    batch = ab.tree_batch([50, 40], [[-1, 0, 0], [-1, 0]], table, 16, "cuda", [1, 0])
    X = normal(2, 5, block.hidden, dtype=torch.float32)
    ws = torch.empty(block.workspace_size(5, batch, cache), dtype=torch.uint8, device="cuda") if own else None
    block.step(X, cache, batch, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block.step(X, cache, batch, workspace=ws)
    other = w2.KVCache(torch.zeros(24, 16, block.n_kv, block.head_dim, dtype=torch.bfloat16, device="cuda"),
                       torch.zeros(24, 16, block.n_kv, block.head_dim, dtype=torch.bfloat16, device="cuda"))
    large = ab.causal_batch([0, 0], [150, 140], table, 16, "cuda", [0, 1])
    for i in range(4):
        block.step(normal(3 + i, 290, block.hidden, dtype=torch.float32), other, large)
        marks = [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in (1 << 12, 1 << 16, 1 << 20, 1 << 22) for _ in range(3)]
        X.copy_(normal(20 + i, 5, block.hidden, dtype=torch.float32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert all((m == 0x5a).all() for m in marks), f"replay {i} wrote into memory of others"
        assert torch.equal(got, block.step(X, cache, batch)), f"replay {i}"


@pytest.mark.gpu
def test_steps_on_two_streams(w2):
    ab, block, _ = block_and_cache(w2)
    table = torch.arange(20, dtype=torch.int32).view(2, 10).contiguous().cuda()
    batches = [ab.causal_batch([0, 0], n, table, 16, "cuda", [0, 1]) for n in ([150, 140], [33, 71])]
    rows = [normal(1 + i, b.positions.shape[0], block.hidden, dtype=torch.float32) for i, b in enumerate(batches)]
    caches = [w2.KVCache(*(torch.zeros(24, 16, block.n_kv, block.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))) for _ in rows]
    alone = [block.step(x, c, b) for x, c, b in zip(rows, caches, batches)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in rows]
    results = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                results[i].append(block.step(rows[i], caches[i], batches[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, alone[i]) for y in results[i]), f"stream {i}"


# ------------------------------------------------------------------ adapters
P = 4096                                                       # an aligned address that is never followed


def add(w2, base=P, ldb=64, Y=2 * P, ldy=64, act=0, M=3, X=P, adapter=P, rank=None, scale=None):
    lora = w2._LoraStruct(A=P, B=P, rank=rank, scale=scale, a_stride=256 * 16, b_stride=64 * 16, part_end=(ctypes.c_int64 * 4)(64, 0, 0, 0),
                          n_adapters=2, max_rank=16, n_parts=1, gated=0)
    return w2.raw().w2_lora_add(ctypes.byref(lora), 256, 64, X, w2.DT_BF16, 256, M, adapter, base, ldb, Y, ldy, act, P, 1 << 20, None)


def test_adapters_in_place_need_one_stride():
    # rows would be stored over rows that have not been read
    from paper_2508_06753_amd import binding as w2
    assert add(w2, base=P, Y=P, ldb=72, ldy=64) == w2.ERR_INVALID_ARG
    assert add(w2, base=P, Y=P, ldb=64, ldy=128) == w2.ERR_INVALID_ARG
    assert b"stride" in w2.raw().w2_last_error()
    assert add(w2, base=P, Y=P, ldb=72, ldy=64, M=0) == 0


def test_arrays_of_numbers_are_aligned_to_their_types():
    # (the attention's are in test_block_ops.py)
    from paper_2508_06753_amd import binding as w2
    assert add(w2, adapter=P + 2) == add(w2, rank=P + 1) == add(w2, scale=P + 2) == w2.ERR_MISALIGNED
    cache = w2._CacheStruct(k=P, v=P, n_pages=4, page_size=16, k_page_stride=2048, k_slot_stride=128, k_head_stride=64, v_page_stride=2048,
                            v_slot_stride=128, v_head_stride=64, n_heads=2, head_dim=64)
    rope = w2._RopeStruct(P, 64, 0, 1.0)
    for positions, slots in ((P + 2, P), (P, P + 4)):
        assert w2.raw().w2_qk_norm_rope(P, 512, 2, 4, None, None, 0.0, ctypes.byref(rope), positions, 2 * P, 256, ctypes.byref(cache), slots,
                                        None) == w2.ERR_MISALIGNED


@pytest.mark.gpu
@pytest.mark.parametrize("xdt", [torch.float32, torch.bfloat16])
def test_a_workspace_for_many_rows_serves_fewer(w2, xdt):
    """Parts of K are as many as the workspace holds: the size for a program's largest batch is enough for all of them."""
    K, N, n, R = 4096, 256, 5, 64
    lora = w2.Lora(normal(1, n, 2 * R, K, std=0.02), normal(2, n, N, R), gated=True)
    sizes = {M: w2.lora_workspace_size(lora, M) for M in (1, 9, 40, 300, 1200, 4000)}
    assert max(sizes.values()) > sizes[4000], "the case is about sizes that fall"
    ws = torch.full((sizes[4000],), 0xff, dtype=torch.uint8, device="cuda")
    for M in sizes:
        rng = np.random.default_rng(M)
        X, base, ad = normal(3, M, K, dtype=xdt), normal(4, M, N), rng.integers(-1, n, M).astype(np.int32)
        for room in (ws, ws[:(M * 2 * R * 4 + 255) // 256 * 256]):  # (the least: one part)
            Y = w2.lora_add(lora, X, i32(ad), base, workspace=room)
            rows = rng.permutation(M)[:40]
            ref, mag = want.lora(f64(X)[rows], f64(lora.A), f64(lora.B), ad[rows], f64(base)[rows], None, None, np.arange(N) // 16 % 2, 0)
            near(f64(Y)[rows], ref, U * np.abs(ref) + 2.0 ** -13 * mag, f"{M} rows in {room.numel()} bytes")
        if M * 2 * R * 4 > 256:
            with pytest.raises(w2.W2Error):
                w2.lora_add(lora, X, i32(ad), base, workspace=ws[:M * 2 * R * 4 - 256])


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 20, 150])
@pytest.mark.parametrize("xdt", [torch.float32, torch.bfloat16])
def test_infinite_rows_stay_infinite(w2, M, xdt):
    """Row 0 has an infinity where all factors are positive: T is +infinity, and Y has the sign of B."""
    K, N, R = 512, 96, 8
    X, A, B, base = normal(1, M, K, dtype=xdt), normal(2, 1, R, K, std=0.05), normal(3, 1, N, R), normal(4, M, N)
    A[:, :, 5] = A[:, :, 5].abs() + 0.01
    B = (B.abs() + 0.01) * (1 - 2 * (torch.arange(N, device="cuda") % 2))[:, None]
    B = B.bfloat16().contiguous()
    lora, ad = w2.Lora(A, B), torch.zeros(M, dtype=torch.int32, device="cuda")
    clean = w2.lora_add(lora, X, ad, base)
    X[0, 5] = float("inf")
    Y = w2.lora_add(lora, X, ad, base)
    assert torch.equal(Y[1:], clean[1:]), "the other rows"
    assert torch.equal(Y[0].float(), float("inf") * (1.0 - 2 * (torch.arange(N, device="cuda") % 2)))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 20, 150])
def test_largest_numbers_stay_finite(w2, M):
    """Rows, and T, up to the largest fp32 number, which is past the largest of bf16."""
    K, N, R = 512, 96, 8
    X, A, B, base = normal(1, M, K, dtype=torch.float32), normal(2, 1, R, K, std=0.05), normal(3, 1, N, R, std=2.0 ** -100), normal(4, M, N)
    A[:, :, 5] = 1.0
    X[0, 5] = torch.finfo(torch.float32).max                    # T is that, too (the other terms are below its last bit)
    X[M - 1, 5] = -torch.finfo(torch.float32).max
    scale = torch.ones(1, device="cuda")
    ad = np.zeros(M, np.int32)
    ref, mag = want.lora(f64(X), f64(A), f64(B), ad, f64(base), None, [1.0], np.zeros(N, int), 0)
    Y = w2.lora_add(w2.Lora(A, B, scale=scale), X, i32(ad), base)
    near(Y, ref, U * np.abs(ref) + 2.0 ** -13 * mag, f"largest numbers, {M} rows")


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", [0, 2])
@pytest.mark.parametrize("M", [1, 20, 150])
def test_parts_do_not_meet_each_other(w2, gated, act, M):
    """T of one part is past fp32's range: columns of the other parts are what they are."""
    K, R, widths = 512, 16, [32, 16, 48]
    N, P = sum(widths), 2 if gated else 3
    X, A, B, base = normal(1, M, K), normal(2, 1, P * R, K, std=0.05), normal(3, 1, N, R), normal(4, M, N)
    part = np.arange(N) // 16 % 2 if gated else np.repeat(np.arange(P), widths)
    lora = lambda: w2.Lora(A, B, parts=None if gated else widths, gated=gated)  # noqa: E731
    ad = np.zeros(M, np.int32)
    A[:, :, 7] = 0
    ref, mag = want.lora(f64(X), f64(A), f64(B), ad, f64(base), None, None, part, act)
    X[:, 7] = 1e38
    A[:, R:2 * R, 7] = 100.0                                     # part 1: infinite; the others: zero times 1e38
    Y = f64(w2.lora_add(lora(), X, i32(ad), base, act=act))
    out_part = part.reshape(-1, 2, 16)[:, 0].reshape(-1) if act == 2 else part
    other = part.reshape(-1, 2, 16)[:, 1].reshape(-1) if act == 2 else part
    keep = (out_part != 1) & (other != 1)
    near(Y[:, keep], ref[:, keep], (U * np.abs(ref) + 2.0 ** -13 * mag)[:, keep], f"gated {gated}, act {act}, {M} rows")
    if act == 0:
        assert not np.isfinite(Y[:, ~keep]).any()


# ------------------------------------------------------------------ attention
class Requests:
    """Requests of (keys, drafted tokens) over a cache whose pages are in some order; the oracle's view of them."""

    def __init__(self, w2, requests, hq, hkv, D, page=16, seed=0, masks=None, scale=None):
        self.w2, self.requests, self.hq, self.hkv, self.D, self.page = w2, requests, hq, hkv, D, page
        self.scale = D ** -0.5 if scale is None else scale
        rng = np.random.default_rng(seed)
        need = [(n + page - 1) // page for n, _ in requests]
        self.pages, self.M = sum(need) + 1, sum(t for _, t in requests)
        order = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((len(requests), max(need)), -1, np.int32)
        self.starts = np.concatenate([[0], np.cumsum([t for _, t in requests])])
        for r, c in enumerate(need):
            self.table[r, :c] = order[sum(need[:r]):sum(need[:r + 1])]
        self.k, self.v = normal(seed + 1, self.pages, page, hkv, D), normal(seed + 2, self.pages, page, hkv, D)
        self.q = normal(seed + 3, self.M, hq, D, std=1.5)
        self.mask = None
        if masks is not None:
            words = max(m.shape[1] for m in masks)
            self.mask = np.zeros((self.M, words), np.uint64)
            for r, m in enumerate(masks):
                self.mask[self.starts[r]:self.starts[r + 1], :m.shape[1]] = m

    def place(self, r, c):
        return int(self.table[r, c // self.page]), c % self.page

    def run(self, split=True, max_len=None, cols=None, lse=True, kv_len=None):
        w2 = self.w2
        cache = w2.KVCache(self.k, self.v)
        most_t = max(t for _, t in self.requests)
        most_n = max(n for n, _ in self.requests) if max_len is None else max_len
        ws = None
        if split:
            size = w2.tree_attention_workspace_size(len(self.requests), self.M, self.hq, cache, most_t, most_n)
            ws = torch.full((max(16, size),), 0xff, dtype=torch.uint8, device="cuda")
        out = torch.full((self.M, self.hq, self.D), 7.0, dtype=torch.bfloat16, device="cuda")
        L = torch.full((self.M, self.hq), 9.0, device="cuda")
        table = i32(self.table if cols is None else self.table[:, :cols])
        w2.tree_attention(self.q, cache, table, i32(self.starts), i32([n for n, _ in self.requests] if kv_len is None else kv_len), most_t, most_n,
                          mask=None if self.mask is None else torch.tensor(self.mask.view(np.int64), device="cuda"),
                          scale=self.scale, out=out, lse=L, workspace=ws)
        return f64(out), f64(L)

    def oracle(self, r, clip=None):
        """One request's (out, lse, magnitude of the terms, largest score's terms); `clip`: keys from there on are left out."""
        n, t = self.requests[r]
        c = np.arange(n)
        p = self.table[r, c // self.page]
        k, v = f64(self.k)[p, c % self.page], f64(self.v)[p, c % self.page]
        if clip is not None:
            k[clip:] = np.nan
        rows = slice(self.starts[r], self.starts[r + 1])
        return want.attention(f64(self.q)[rows], k, v, t, None if self.mask is None else self.mask[rows], self.scale)

    def check(self, got, what, clip=None):
        out, lse = got
        for r in range(len(self.requests)):
            ref, ref_l, mag, big = self.oracle(r, clip)
            rows = slice(self.starts[r], self.starts[r + 1])
            near(out[rows], ref, U * np.abs(ref) + 2 * U * mag, f"{what}, request {r}")
            empty = np.isinf(ref_l)
            assert np.array_equal(np.isneginf(lse[rows]), empty), f"{what}, request {r}: rows that see nothing"
            near(lse[rows][~empty], ref_l[~empty], (self.D + 8) * 2.0 ** -24 * big + 2.0 ** -18, f"{what}, request {r} lse")


# heads, drafted tokens: the kernel for few rows (eight waves, four, two row tiles), the one for many
FEW = [(8, 8, 64, 1), (8, 2, 128, 3), (8, 2, 128, 7), (4, 2, 256, 5)]
MANY = [(8, 2, 128, 12), (8, 2, 64, 70), (8, 2, 256, 40), (6, 2, 96, 40)]


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D,t", FEW + MANY)
@pytest.mark.parametrize("masked", [False, True])
def test_keys_past_the_limits_are_left_out(w2, hq, hkv, D, t, masked):
    """kv_len above max_len, and above what the page table covers: the first keys, seen as if the others were there."""
    rng = np.random.default_rng(t)
    for n, page in ((300, 16), (1500, 16), (300, 24)):
        for clip in (192, 288 if n == 300 else 1488, n - t):       # before the drafted tokens, among them, all of them away
            clip = min(clip, n) // page * page
            c = Requests(w2, [(n, t), (60, min(t, 60))], hq, hkv, D, page=page, seed=n + t, masks=[tree_masks(t, rng), tree_masks(min(t, 60), rng)] if masked else None)
            c.check(c.run(max_len=clip), f"max_len {clip} of {n}, {t} tokens", clip)
            c.check(c.run(cols=clip // page), f"{clip // page} pages of {page}, {n} keys, {t} tokens", clip)
            c.check(c.run(cols=clip // page, split=False), f"{clip // page} pages of {page}, {n} keys, {t} tokens, one workgroup", clip)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D,t", FEW + MANY)
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_queries_and_keys_that_are_not_finite_show(w2, hq, hkv, D, t, split, bad):
    """A query with NaN or an infinity has no finite scores' softmax: its head's row is NaN, all others are as they were.  The same
    of a key for the rows that see it."""
    for n in (90, 1400):
        c = Requests(w2, [(n, t), (50, 1)], hq, hkv, D, seed=n + t)
        clean, clean_l = c.run(split)
        c.check((clean, clean_l), f"{n} keys, {t} tokens")
        row, head = t // 2, hq - 1
        kept = c.q[row, head, 3].clone()
        c.q[row, head, 3] = bad
        out, lse = c.run(split)
        assert np.isnan(out[row, head]).all() and np.isnan(lse[row, head]), f"{n} keys, {t} tokens: a row without a finite score"
        out[row, head], lse[row, head] = clean[row, head], clean_l[row, head]
        assert np.array_equal(out, clean) and np.array_equal(lse, clean_l), f"{n} keys, {t} tokens: the other rows"
        c.q[row, head, 3] = kept
        # the last drafted token's key: only the last row sees it
        c.k[c.place(0, n - 1) + (hkv - 1, 5)] = float("nan")
        out, lse = c.run(split)
        hit = np.zeros(lse.shape, bool)
        hit[t - 1, hq - hq // hkv:] = True
        assert np.isnan(out[hit]).all() and np.isnan(lse[hit]).all(), f"{n} keys, {t} tokens: rows that see a key of NaN"
        assert np.array_equal(out[~hit], clean[~hit]) and np.array_equal(lse[~hit], clean_l[~hit])


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D,t", FEW + MANY)
@pytest.mark.parametrize("split", [False, True])
def test_values_that_are_not_finite_show(w2, hq, hkv, D, t, split):
    """A committed value that is NaN or infinite: that number of the outputs of its heads, and nothing else."""
    for n in (90, 1400):
        c = Requests(w2, [(n, t), (50, 1)], hq, hkv, D, seed=n + t)
        clean, clean_l = c.run(split)
        for at in (0, n - t - 1):
            for bad in (float("nan"), float("inf")):
                where = c.place(0, at) + (hkv - 1, D - 2)
                kept = c.v[where].clone()
                c.v[where] = bad
                out, lse = c.run(split)
                c.v[where] = kept
                hit = np.zeros(out.shape, bool)
                hit[:t, hq - hq // hkv:, D - 2] = True
                assert not np.isfinite(out[hit]).any(), f"{n} keys, {t} tokens, value of key {at}"
                assert np.array_equal(out[~hit], clean[~hit]) and np.array_equal(lse, clean_l)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D,t", [h for h in FEW + MANY if h[3] > 1] + [(2, 2, 64, 100)])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("page", [16, 24])
def test_drafted_tokens_that_no_row_sees_may_hold_anything(w2, hq, hkv, D, t, split, page):
    """A tree that is filled up to its size: tokens that are not there, whose keys and values were never written."""
    rng = np.random.default_rng(t)
    for n in (t, t + 77, 1400):
        for hidden in ([0], [t - 1], list(range(t // 2, t)), list(range(0, t, 2)), list(range(t))):
            own = tree_masks(t, rng)
            for j in hidden:
                own[:, j // 64] &= ~np.uint64(1 << (j % 64))
            c = Requests(w2, [(n, t), (50, 1)], hq, hkv, D, page=page, seed=n + t, masks=[own, tree_masks(1, rng)])
            ref = [c.oracle(r) for r in range(2)]
            for j in hidden:
                p, at = c.place(0, n - t + j)
                c.k[p, at], c.v[p, at] = float("nan"), float("inf") if j % 2 else float("nan")
            out, lse = c.run(split)
            for r in range(2):
                rows = slice(c.starts[r], c.starts[r + 1])
                o, l, mag, big = ref[r]
                what = f"{n} keys, {t} tokens, hidden {hidden[:3]}, request {r}"
                near(out[rows], o, U * np.abs(o) + 2 * U * mag, what)
                empty = np.isinf(l)
                assert np.array_equal(np.isneginf(lse[rows]), empty), what
                near(lse[rows][~empty], l[~empty], (D + 8) * 2.0 ** -24 * big + 2.0 ** -18, what + " lse")


@pytest.mark.gpu
def test_drafted_tokens_past_the_mask_may_hold_anything(w2):
    # one word of mask, a hundred tokens: the last 36 are seen by nobody
    own = tree_masks(100, np.random.default_rng(1))[:, :1].copy()
    for hq, hkv, D in ((2, 2, 64), (4, 1, 128)):
        c = Requests(w2, [(300, 100)], hq, hkv, D, masks=[own])
        o, l, mag, _ = c.oracle(0)
        for j in range(64, 100):
            p, at = c.place(0, 200 + j)
            c.k[p, at] = c.v[p, at] = float("nan")
        out, _ = c.run()
        near(out, o, U * np.abs(o) + 2 * U * mag, "mask of one word")


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D", [(8, 2, 128), (8, 2, 64), (6, 2, 96), (4, 2, 256)])
def test_single_tokens_agree_with_the_rows_of_a_chunk(w2, hq, hkv, D):
    """The two kernels with each other: rows of a causal chunk, and each as the single token behind its predecessors."""
    n, t = 500, 50
    c = Requests(w2, [(n, t)], hq, hkv, D, seed=3)
    out, lse = c.run()
    c.check((out, lse), "chunk")
    _, _, mag, big = c.oracle(0)
    for i in (t - 1, 0, 17):
        kept, c.requests, c.M, c.starts, q = c.requests, [(n - t + 1 + i, 1)], 1, [0, 1], c.q
        c.q = q[i:i + 1]
        one, one_l = c.run()
        c.requests, c.M, c.starts, c.q = kept, t, [0, t], q
        # both within the bounds of the oracle: twice them of each other
        near(one[0], out[i], 2 * U * np.abs(out[i]) + 4 * U * mag[i], f"row {i}")
        near(one_l[0], lse[i], 2 * ((D + 8) * 2.0 ** -24 * big + 2.0 ** -18), f"row {i} lse")


def one_part(q, k, v, t, scale):
    """Causal attention whose weights are rounded to bf16 once before they meet v: what the bound below has to notice."""
    T, hq, D = q.shape
    out = np.zeros((T, hq, D))
    for i in range(T):
        n = k.shape[0] - t + i + 1
        for h in range(hq):
            kv = h * k.shape[1] // hq
            s = scale * (k[:n, kv] @ q[i, h])
            p = np.exp(s - s.max())
            out[i, h] = f64(torch.tensor(p).bfloat16()) @ v[:n, kv] / p.sum()
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D,t", FEW)
@pytest.mark.parametrize("split", [False, True])
def test_few_rows_hold_weights_in_sixteen_bits(w2, hq, hkv, D, t, split):
    """The kernel for few rows multiplies weights in two bf16 parts: one rounding of the output, and of the terms 2^-16 for
    the parts (2^-8 of 2^-8), 2^-18 of sums and exponentials, and twice the scores' own error, (D + 8) 2^-24 of their
    terms.  Weights in one part leave that bound where keys are few."""
    for n in (t + 2, t + 11, 70):
        c = Requests(w2, [(n, t)] * 3, hq, hkv, D, seed=n + t)
        out, _ = c.run(split)
        noticed = 0
        for r in range(3):
            ref, _, mag, big = c.oracle(r)
            rows = slice(c.starts[r], c.starts[r + 1])
            bound = U * np.abs(ref) + (2.0 ** -16 + 2.0 ** -18 + 2 * (D + 8) * 2.0 ** -24 * big) * mag
            near(out[rows], ref, bound, f"{n} keys, {t} tokens")
            at = np.arange(n)
            k, v = (f64(x)[c.table[r, at // c.page], at % c.page] for x in (c.k, c.v))
            once = f64(torch.tensor(one_part(f64(c.q)[rows], k, v, t, c.scale)).bfloat16())
            noticed += np.count_nonzero(np.abs(once - ref) > bound)
        assert noticed > 0


def plain_causal(q, k, v, n_drafted, scale):
    """want.attention without a mask, for many rows at once: (out, lse, terms' magnitude, largest score's terms)."""
    T, hq, D = q.shape
    L, hkv, _ = k.shape
    seen = np.arange(L)[None, :] <= np.arange(T)[:, None] + (L - n_drafted)
    out, mag, lse, big = np.zeros((T, hq, D)), np.zeros((T, hq, D)), np.zeros((T, hq)), 0.0
    for h in range(hq):
        kk, vv = k[:, h * hkv // hq], v[:, h * hkv // hq]
        s = np.where(seen, scale * (q[:, h] @ kk.T), -np.inf)
        big = max(big, float(np.max(np.abs(scale) * (np.abs(q[:, h]) @ np.abs(kk).T))))
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(1, keepdims=True)
        lse[:, h] = (top + np.log(total))[:, 0]
        out[:, h], mag[:, h] = p / total @ vv, p / total @ np.abs(vv)
    return out, lse, mag, big


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,D,t,n", [(8, 1, 64, 1501, 1501), (16, 1, 128, 700, 1900), (32, 4, 128, 333, 333), (6, 2, 96, 901, 1203)])
def test_prompts_of_many_row_tiles(w2, hq, hkv, D, t, n):
    c = Requests(w2, [(n, t)], hq, hkv, D, seed=t)
    at = np.arange(n)
    k, v = (f64(x)[c.table[0, at // 16], at % 16] for x in (c.k, c.v))
    ref, ref_l, mag, big = plain_causal(f64(c.q), k, v, t, c.scale)
    few = want.attention(f64(c.q)[:1], k[:n - t + 1], v[:n - t + 1], 1, None, c.scale)[0]
    assert np.abs(few - ref[:1]).max() < 1e-12
    out, lse = c.run()
    near(out, ref, U * np.abs(ref) + 2 * U * mag, f"{t} tokens")
    near(lse, ref_l, (D + 8) * 2.0 ** -24 * big + 2.0 ** -18, f"{t} tokens, lse")


# ------------------------------------------------------------------ norm, rotation, cache
@pytest.mark.gpu
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rd", [(128, 96), (64, 0), (24, 12), (80, 60), (256, 4), (96, 72), (128, 64)])
def test_numbers_that_are_not_rotated_meet_no_others(w2, D, rd, inter):
    """Past the rotated part a number stays what it is, and so do its neighbours when it is NaN or infinite."""
    M, hq, hkv = 5, 3, 2
    x = normal(D + rd, M, (hq + 2 * hkv) * D)
    y = x.view(M, -1, D)
    for m in range(M):
        for h in range(hq + hkv):
            at = rd + (7 * m + 3 * h) % (D - rd)
            y[m, h, at] = (float("inf"), float("nan"), -float("inf"))[(m + h) % 3]
    clean = torch.where(torch.isfinite(y), y, torch.ones_like(y)).contiguous()
    rope = w2.Rope(rd, interleaved=inter) if rd else None
    pos = torch.arange(100, 100 + M, dtype=torch.int32, device="cuda")
    results = []
    for t in (x, clean.view(M, -1)):
        k, v = (torch.zeros(1, 8, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q = w2.qk_norm_rope(t, hq, rope, pos, w2.KVCache(k, v))
        results.append(torch.cat((q, k[0, :M]), 1))
    got, ref = results
    bad = ~torch.isfinite(y[:, :hq + hkv])
    assert torch.equal(got[~bad], ref[~bad]), "a neighbour changed"
    assert torch.equal(torch.nan_to_num(got[bad]), torch.nan_to_num(y[:, :hq + hkv][bad])), "a number that is not finite changed"
    assert torch.equal(torch.isnan(got[bad]), torch.isnan(y[:, :hq + hkv][bad]))
