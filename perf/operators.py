"""The operators around the projections of an attention block, as cases that can be timed and checked.

* ``rope``: norms of queries and keys, rotary positions, keys and values into the paged cache: one pass over the rows
  that the QKV projection wrote.
* ``lora``: low-rank adapters of many requests added beside a shared projection, with its activation.
* ``tree``: attention of every request's drafted tokens over its pages of the cache; one drafted token is plain
  decoding, no mask is a causal chunk of a prompt.

A plain form in elementary torch operations, in 32 bits, stands beside each: `own` chooses.  Head counts, projections
and group sizes are those of the shapes that the benchmark runs (2048, 4096 and 5120 columns) and generic ones.
Lengths of requests, drafted tokens per request, ranks and the adapters' shares of the rows depend on a case's sizes
alone; values, pages, trees and the order of the rows depend on the seed.
"""
import math

import numpy as np
import torch

own = False


def listed():
    return [
        # one new token of one user, 8B-class heads: latency
        dict(name="rope_m1", op="rope", m=1, hq=32, hkv=8, d=128, rd=128, pairs=False, norm=True, base=500000.0,
             factor=8.0, mscale=1.0, original=8192, top=131072, page=16),
        # drafted tokens of a batch, a quarter of the head not rotated, pairs side by side, no norm
        dict(name="rope_m96_partial_pairs", op="rope", m=96, hq=40, hkv=8, d=128, rd=96, pairs=True, norm=False,
             base=10000.0, factor=1.0, mscale=1.0, original=4096, top=4096, page=64),
        # a prompt of odd length at the end of a long context, scaled frequencies and amplitude
        dict(name="rope_m8191_long", op="rope", m=8191, hq=40, hkv=8, d=128, rd=128, pairs=False, norm=True,
             base=1000000.0, factor=4.0, mscale=1.1386294361119891, original=32768, top=131072, page=32),
        # one new token of one user on the smallest fused QKV projection with one adapter: latency
        dict(name="lora_m1_qkv", op="lora", m=1, k=4096, n=6144, parts="4096,1024,1024", rank=16, adapters=1,
             mixed_ranks=False, none=False, order="mixed", x="bf16", act="none"),
        # a batch of users, nearly each with an adapter of its own, some with none, ranks of many sizes
        dict(name="lora_m61_many", op="lora", m=61, k=5120, n=7168, parts="5120,1024,1024", rank=32, adapters=48,
             mixed_ranks=True, none=True, order="mixed", x="bf16", act="none"),
        # the same on a deep projection from rows in 32 bits, an odd rank
        dict(name="lora_m37_down_f32", op="lora", m=37, k=14336, n=4096, parts="4096", rank=40, adapters=9,
             mixed_ranks=False, none=False, order="mixed", x="f32", act="none"),
        # prompts of a few users through the gated projection
        dict(name="lora_m4000_gated", op="lora", m=4000, k=4096, n=28672, parts="gated", rank=64, adapters=5,
             mixed_ranks=False, none=False, order="runs", x="bf16", act="silu_mul"),
        # one user, one token, a short conversation: latency
        dict(name="tree_r1_t1_short", op="tree", requests=1, drafted=1, length=700, hq=32, hkv=8, d=128, page=16,
             masked=False),
        # continuous batching: one token each, conversations of very different lengths
        dict(name="tree_r48_t1", op="tree", requests=48, drafted=1, length=8000, hq=40, hkv=8, d=128, page=64,
             masked=False),
        # speculative decoding of a batch: small trees
        dict(name="tree_r16_t9", op="tree", requests=16, drafted=9, length=4100, hq=32, hkv=8, d=128, page=16,
             masked=True),
        # one user with a long context and a wide tree
        dict(name="tree_r2_t64_long", op="tree", requests=2, drafted=64, length=120000, hq=40, hkv=8, d=128, page=32,
             masked=True),
        # chunks of prompts, heads of 64
        dict(name="tree_r4_t1000_causal", op="tree", requests=4, drafted=1000, length=5000, hq=32, hkv=8, d=64, page=32,
             masked=False),
    ]


# ---------------------------------------------------------------- sizes that follow from a case
def _lengths(case):
    """Keys and drafted tokens of every request: ragged, the first one at the full length."""
    out = []
    for j in range(case["requests"]):
        cut = (j * 0.6180339887) % 1.0
        t = max(1, int(round(case["drafted"] * (1 - 0.5 * cut))))
        out.append((max(t, int(case["length"] * (1 - 0.8 * cut))), t))
    return out


def _row_adapters(case):
    """The adapter of every row, before any shuffling; -1: none."""
    m, na = case["m"], case["adapters"]
    rows = [j * na // m for j in range(m)] if case["order"] == "runs" else [j % na for j in range(m)]
    return [-1 if case["none"] and j % 7 == 3 else a for j, a in enumerate(rows)]


def _ranks(case):
    r = case["rank"]
    return [max(1, r - (5 * j) % r) if case["mixed_ranks"] else r for j in range(case["adapters"])]


def _parts(case):
    """Number of parts of the columns, and the part of every column."""
    n = case["n"]
    if case["parts"] == "gated":                              # blocks of 16 columns: gate, up, gate, up ...
        return 2, [(c // 16) % 2 for c in range(n)]
    widths = [int(w) for w in case["parts"].split(",")]
    return len(widths), [p for p, w in enumerate(widths) for _ in range(w)]


def _phases(case):
    """Turns per position of every rotated pair, as fractions of 2^64, and as floating numbers.

    Frequencies base^(-2i/rd); with a factor, those whose wavelength leaves less than one turn in the original context
    are divided by it, those with more than 32 turns stay, a straight line in the turns between."""
    rd = case["rd"]
    freq = []
    for i in range(rd // 2):
        f = case["base"] ** (-2.0 * i / rd) / (2 * math.pi)
        if case["factor"] != 1.0:
            stay = min(1.0, max(0.0, (case["original"] * f - 1.0) / 31.0))
            f = f * stay + f / case["factor"] * (1.0 - stay)
        freq.append(f)
    return freq


# ---------------------------------------------------------------- drawn cases
def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


HEADS = [(32, 8, 128), (40, 8, 128), (64, 8, 128), (8, 4, 256), (32, 8, 64), (12, 12, 64), (15, 5, 96), (16, 1, 128),
         (16, 16, 128), (21, 3, 80)]


def _draw_once(rng):
    op = rng.choice(["rope", "lora", "tree", "lora", "tree", "tree"])
    if op == "rope":
        hq, hkv, d = rng.choice(HEADS)
        m = _log(rng, 1, 8191)
        factor = rng.choice([1.0, 2.0, 4.0, 8.0])
        return dict(op=op, m=m, hq=hq, hkv=hkv, d=d, rd=rng.choice([d, d, d // 2, d // 4 * 3]), pairs=rng.random() < 0.5,
                    norm=rng.random() < 0.6, base=rng.choice([10000.0, 500000.0, 1000000.0]), factor=factor,
                    mscale=0.1 * math.log(factor) + 1.0, original=rng.choice([4096, 8192, 32768]),
                    top=_log(rng, max(m, 2048), 131072), page=rng.choice([16, 32, 64, 48, 1]))
    if op == "lora":
        k, n, parts = rng.choice([(2048, 2048, "2048"), (4096, 6144, "4096,1024,1024"), (4096, 4096, "4096"),
                                  (4096, 28672, "gated"), (14336, 4096, "4096"), (5120, 7168, "5120,1024,1024"),
                                  (5120, 34816, "gated"), (17408, 5120, "5120"), (1280, 1048, "640,408")])
        m = _log(rng, 1, 4000)
        return dict(op=op, m=m, k=k, n=n, parts=parts, rank=rng.choice([8, 16, 32, 64, 24, 128]),
                    adapters=_log(rng, 1, 64), mixed_ranks=rng.random() < 0.4, none=rng.random() < 0.4,
                    order=rng.choice(["runs", "mixed"]) if m <= 256 else "runs", x=rng.choice(["bf16", "bf16", "f32"]),
                    act="silu_mul" if parts == "gated" and rng.random() < 0.7 else "none")
    hq, hkv, d = rng.choice(HEADS)
    kind = rng.choice(["one", "tree", "tree", "chunk"])
    drafted = 1 if kind == "one" else rng.randint(2, 64) if kind == "tree" else _log(rng, 65, 1024)
    return dict(op=op, requests=_log(rng, 1, 64), drafted=drafted, length=_log(rng, max(8, drafted), 120000), hq=hq, hkv=hkv,
                d=d, page=rng.choice([16, 32, 64, 48, 1]), masked=kind == "tree")


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), _cost(c))
    while True:
        case = _draw_once(rng)
        # what the plain form needs in memory is bounded as well: padded keys, scores, factors of every adapter
        if _cost(case) > most[case["op"]]:
            continue
        if case["op"] == "tree" and (case["requests"] * case["length"] * case["hkv"] * case["d"] > 1 << 30 or
                                     case["requests"] * case["drafted"] * case["hq"] * case["length"] > 1 << 30):
            continue
        if case["op"] == "lora" and (case["adapters"] * case["rank"] * max(case["m"], case["n"]) > 1 << 28 or
                                     case["m"] * case["adapters"] * case["rank"] * (3 * case["k"] + case["n"]) > 1 << 43):
            continue
        return case


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = {"case": case}
    return {"rope": _prepare_rope, "lora": _prepare_lora, "tree": _prepare_tree}[case["op"]](s, case, gen, rng)


def _normal(gen, *shape, dtype=torch.bfloat16, std=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _ints(values, dtype):
    return torch.tensor(np.asarray(values), dtype=dtype, device="cuda")


def _prepare_rope(s, case, gen, rng):
    m, hq, hkv, d, page = (case[k] for k in ("m", "hq", "hkv", "d", "page"))
    s["x"] = _normal(gen, m, (hq + 2 * hkv) * d)
    if case["norm"]:
        s["qw"] = (1.0 + _normal(gen, d, dtype=torch.float32, std=0.2)).bfloat16()
        s["kw"] = (1.0 + _normal(gen, d, dtype=torch.float32, std=0.2)).bfloat16()
    else:
        s["qw"] = s["kw"] = None
    # a run of positions at the end of a context for prompts, anything for the tokens of a batch
    pos = np.arange(case["top"] - m, case["top"]) if m > 512 else rng.integers(0, case["top"], m)
    s["positions"] = _ints(pos, torch.int32)
    pages = (m + page - 1) // page + 3
    slots = rng.permutation(pages)[:, None] * page + np.arange(page)[None, :]
    s["slots"] = _ints(slots.reshape(-1)[:m], torch.int64)
    s["k_cache"] = _normal(gen, pages, page, hkv, d)
    s["v_cache"] = _normal(gen, pages, page, hkv, d)
    freq = _phases(case)
    s["phase"] = _ints([(int(f * 2.0 ** 64) + (1 << 63)) % (1 << 64) - (1 << 63) for f in freq], torch.int64)
    if own:
        from paper_2508_06753_amd import binding as w2
        scaling = None if case["factor"] == 1.0 else ("bands", case["factor"], case["original"], 1.0, 32.0)
        s["w2"] = w2
        s["rope"] = w2.Rope(case["rd"], base=case["base"], interleaved=case["pairs"], scaling=scaling,
                            mscale=case["mscale"])
        s["cache"] = w2.KVCache(s["k_cache"], s["v_cache"])
        s["q"] = torch.empty((m, hq, d), dtype=torch.bfloat16, device="cuda")
    return s


def _prepare_lora(s, case, gen, rng):
    m, k, n, r, na = (case[x] for x in ("m", "k", "n", "rank", "adapters"))
    parts, of_column = _parts(case)
    s["x"] = _normal(gen, m, k, dtype=torch.float32 if case["x"] == "f32" else torch.bfloat16)
    s["a"] = _normal(gen, na, parts * r, k, std=1.0 / math.sqrt(k))
    s["b"] = _normal(gen, na, n, r, std=0.5 / math.sqrt(r))
    s["base"] = _normal(gen, m, n)
    s["rank"] = _ints(_ranks(case), torch.int32)
    s["scale"] = torch.empty(na, dtype=torch.float32, device="cuda").uniform_(0.5, 2.0, generator=gen)
    rows = np.asarray(_row_adapters(case))
    s["adapter"] = _ints(rng.permutation(rows) if case["order"] == "mixed" else rows, torch.int32)
    s["columns"] = [_ints([c for c, q in enumerate(of_column) if q == p], torch.int64) for p in range(parts)]
    if own:
        from paper_2508_06753_amd import binding as w2
        s["w2"] = w2
        gated = case["parts"] == "gated"
        s["lora"] = w2.Lora(s["a"], s["b"], rank=s["rank"], scale=s["scale"], gated=gated,
                            parts=None if gated else [int(w) for w in case["parts"].split(",")])
        s["act"] = w2.ACT_SILU_MUL if case["act"] == "silu_mul" else w2.ACT_NONE
        s["workspace"] = torch.empty(w2.lora_workspace_size(s["lora"], m), dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty((m, n // 2 if case["act"] == "silu_mul" else n), dtype=torch.bfloat16, device="cuda")
    return s


def _prepare_tree(s, case, gen, rng):
    hq, hkv, d, page = (case[k] for k in ("hq", "hkv", "d", "page"))
    lengths = _lengths(case)
    rows = sum(t for _, t in lengths)
    s["max_rows"], s["max_len"] = max(t for _, t in lengths), max(n for n, _ in lengths)
    s["total_len"] = sum(n for n, _ in lengths)
    need = [(n + page - 1) // page for n, _ in lengths]
    pages = sum(need) + 2
    order = rng.permutation(pages)
    table = np.zeros((len(lengths), max(need)), np.int32)
    at = 0
    for j, c in enumerate(need):
        table[j, :c] = order[at:at + c]
        at += c
    s["table"] = _ints(table, torch.int32)
    s["q"] = _normal(gen, rows, hq, d, std=2.0)
    s["k_cache"] = _normal(gen, pages, page, hkv, d)
    s["v_cache"] = _normal(gen, pages, page, hkv, d)
    s["row_start"] = _ints(np.concatenate([[0], np.cumsum([t for _, t in lengths])]), torch.int32)
    s["kv_len"] = _ints([n for n, _ in lengths], torch.int32)
    s["mask"] = None
    if case["masked"]:                                        # random trees: every token sees its ancestors and itself
        bits = []
        for _, t in lengths:
            seen = []
            for i in range(t):
                parent = int(rng.integers(max(-1, i - 6), i)) if i else -1
                seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
            bits += seen
        s["mask"] = _ints([b - (1 << 64) if b >> 63 else b for b in bits], torch.int64).view(-1, 1)
    if own:
        from paper_2508_06753_amd import binding as w2
        s["w2"] = w2
        s["cache"] = w2.KVCache(s["k_cache"], s["v_cache"])
        size = w2.tree_attention_workspace_size(len(lengths), rows, hq, s["cache"], s["max_rows"], s["max_len"],
                                                s["total_len"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty((rows, hq, d), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty((rows, hq), dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    return {"rope": _plain_rope, "lora": _plain_lora, "tree": _plain_tree}[state["case"]["op"]](state, state["case"])


def _run_own(s):
    w2, case = s["w2"], s["case"]
    if case["op"] == "rope":
        q = w2.qk_norm_rope(s["x"], case["hq"], s["rope"], s["positions"], s["cache"], s["slots"], q_weight=s["qw"],
                            k_weight=s["kw"], eps=1e-6, out=s["q"])
        return q, s["k_cache"], s["v_cache"]
    if case["op"] == "lora":
        return w2.lora_add(s["lora"], s["x"], s["adapter"], s["base"], act=s["act"], out=s["out"],
                           workspace=s["workspace"])
    out = w2.tree_attention(s["q"], s["cache"], s["table"], s["row_start"], s["kv_len"], s["max_rows"], s["max_len"],
                            mask=s["mask"], total_len=s["total_len"], out=s["out"], lse=s["lse"],
                            workspace=s["workspace"])
    return out, s["lse"]


def _plain_rope(s, case):
    m, hq, hkv, d, rd = (case[k] for k in ("m", "hq", "hkv", "d", "rd"))
    x = s["x"].float().view(m, hq + 2 * hkv, d)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], s["x"].view(m, -1, d)[:, hq + hkv:]
    if case["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-6) * s["qw"].float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-6) * s["kw"].float()
    # whole turns drop out of the 64-bit product
    turns = (s["positions"].long()[:, None] * s["phase"][None, :]) >> 32
    angle = turns.float() * (2 * math.pi / 2 ** 32)
    cos, sin = (torch.cos(angle) * case["mscale"])[:, None], (torch.sin(angle) * case["mscale"])[:, None]

    def rotate(t):
        head, rest = t[..., :rd], t[..., rd:]
        a, b = (head[..., 0::2], head[..., 1::2]) if case["pairs"] else (head[..., :rd // 2], head[..., rd // 2:])
        a, b = a * cos - b * sin, b * cos + a * sin
        head = torch.stack((a, b), -1).flatten(-2) if case["pairs"] else torch.cat((a, b), -1)
        return torch.cat((head, rest), -1).bfloat16()

    s["k_cache"].view(-1, hkv, d)[s["slots"]] = rotate(k)
    s["v_cache"].view(-1, hkv, d)[s["slots"]] = v
    return rotate(q), s["k_cache"], s["v_cache"]


def _plain_lora(s, case):
    m, n, r, na = (case[x] for x in ("m", "n", "rank", "adapters"))
    parts = len(s["columns"])
    # every row against every adapter, then the row's own one is kept
    t = (s["x"].float() @ s["a"].float().view(na * parts * r, -1).t()).view(m, na, parts, r)
    which = torch.arange(na, device="cuda")
    keep = (s["adapter"].long()[:, None] == which).float() * s["scale"]
    inside = (torch.arange(r, device="cuda")[None, :] < s["rank"][:, None]).float()
    t = t * keep[:, :, None, None] * inside[None, :, None, :]
    b = s["b"].float().permute(0, 2, 1).reshape(na * r, n)
    z = s["base"].float()
    for p, columns in enumerate(s["columns"]):
        z[:, columns] += t[:, :, p].reshape(m, na * r) @ b[:, columns]
    if case["act"] == "silu_mul":
        z = z.view(m, n // 32, 2, 16)
        z = (z[:, :, 0] / (1.0 + torch.exp(-z[:, :, 0])) * z[:, :, 1]).reshape(m, n // 2)
    return z.bfloat16()


def _seen(s, device="cuda"):
    """Which keys every padded row of every request sees: [requests, max_rows, max_len], and the rows that exist."""
    start, kv_len = s["row_start"].long(), s["kv_len"].long()
    drafted = (start[1:] - start[:-1])[:, None]
    i = torch.arange(s["max_rows"], device=device)[None, :]
    row = torch.clamp(start[:-1, None] + i, max=s["q"].shape[0] - 1)
    after = torch.arange(s["max_len"], device=device)[None, :] - (kv_len[:, None] - drafted)     # [requests, max_len]
    if s["mask"] is None:
        tail = after[:, None, :] <= i[:, :, None]
    else:
        tail = (s["mask"][row, 0][:, :, None] >> torch.clamp(after, 0, 63)[:, None, :]) & 1 > 0
    seen = ((after < 0)[:, None, :] | tail) & (after < drafted)[:, None, :]
    return seen, row, i < drafted


def _plain_tree(s, case):
    hq, hkv, d, page = (case[k] for k in ("hq", "hkv", "d", "page"))
    g, r, t, most = hq // hkv, case["requests"], s["max_rows"], s["max_len"]
    seen, row, exists = _seen(s)
    at = torch.arange(most, device="cuda")
    slot = s["table"].long()[:, at // page] * page + at % page                                    # [requests, max_len]
    k = s["k_cache"].view(-1, hkv, d)[slot].permute(0, 2, 1, 3).float()                            # [r, hkv, max_len, d]
    q = s["q"][row].float().view(r, t, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(r, hkv, t * g, d)
    score = (torch.matmul(q, k.transpose(2, 3)) / math.sqrt(d)).view(r, hkv, t, g, most)
    del k
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = s["v_cache"].view(-1, hkv, d)[slot].permute(0, 2, 1, 3).float()
    out = torch.matmul(p.view(r, hkv, t * g, most), v).view(r, hkv, t, g, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    lse = (top + torch.log(total))[..., 0]
    out = out.permute(0, 2, 1, 3, 4).reshape(r, t, hq, d)
    lse = lse.permute(0, 2, 1, 3).reshape(r, t, hq)
    start = s["row_start"].long()
    m = s["q"].shape[0]
    request = torch.bucketize(torch.arange(m, device="cuda"), start[1:], right=True)
    inside = torch.arange(m, device="cuda") - start[request]
    return out[request, inside].bfloat16(), lse[request, inside]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "rope":
        m, heads = case["m"], case["hq"] + 2 * case["hkv"]
        turned = m * (case["hq"] + case["hkv"])
        return {"bytes": 4 * m * heads * case["d"] + 12 * m + 8 * case["rd"] // 2,
                "flops": turned * (3 * case["rd"] + (4 * case["d"] if case["norm"] else 0))}
    if case["op"] == "lora":
        m, k, n = case["m"], case["k"], case["n"]
        parts, rows, ranks = _parts(case)[0], _row_adapters(case), _ranks(case)
        used = sum(ranks[a] for a in set(rows) if a >= 0)
        live = sum(ranks[a] for a in rows if a >= 0)
        out = n // 2 if case["act"] == "silu_mul" else n
        return {"bytes": m * k * (4 if case["x"] == "f32" else 2) + 2 * used * (parts * k + n) + 2 * m * (n + out) + 4 * m,
                "flops": 2 * live * (parts * k + n) + m * n}
    lengths = _lengths(case)
    rows = sum(t for _, t in lengths)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    # a masked row sees its context and its ancestors; a causal one all keys up to its own
    pairs = sum(t * (n - t) + (t if case["masked"] else t * (t + 1) // 2) for n, t in lengths)
    return {"bytes": 4 * hkv * d * sum(n for n, _ in lengths) + 4 * rows * hq * d + 4 * rows * hq + 8 * rows,
            "flops": 4 * hq * d * pairs}


# ---------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return {"rope": _exact_rope, "lora": _exact_lora, "tree": _exact_tree}[case["op"]](s, case)


def _exact_rope(s, case):
    hq, hkv, d, rd = (case[k] for k in ("hq", "hkv", "d", "rd"))
    x = s["x"].double().view(case["m"], -1, d)
    freq = torch.tensor(_phases(case), dtype=torch.float64, device="cuda")
    turns = s["positions"].double()[:, None] * freq
    e = torch.polar(torch.full_like(turns, case["mscale"]), 2 * math.pi * (turns - torch.floor(turns)))[:, None]

    def side(t, w):
        if w is not None:
            t = t / torch.sqrt((t ** 2).sum(-1, keepdim=True) / d + 1e-6) * w.double()
        t = t.clone()
        first, second = (slice(0, rd, 2), slice(1, rd, 2)) if case["pairs"] else (slice(0, rd // 2), slice(rd // 2, rd))
        turned = torch.complex(t[..., first], t[..., second]) * e
        t[..., first], t[..., second] = turned.real, turned.imag
        return t

    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    k_cache.view(-1, hkv, d).index_copy_(0, s["slots"], side(x[:, hq:hq + hkv], s["kw"]))
    v_cache.view(-1, hkv, d).index_copy_(0, s["slots"], x[:, hq + hkv:].contiguous())
    return side(x[:, :hq], s["qw"]), k_cache, v_cache


def _exact_lora(s, case):
    parts, of_column = _parts(case)
    of_column = torch.tensor(of_column, device="cuda")
    z = s["base"].double()
    for a, rank in enumerate(_ranks(case)):
        rows = (s["adapter"] == a).nonzero()[:, 0]
        if not rows.numel():
            continue
        x = s["x"][rows].double()
        for p in range(parts):
            columns = (of_column == p).nonzero()[:, 0]
            t = x @ s["a"][a, p * case["rank"]:p * case["rank"] + rank].double().t()
            z[rows[:, None], columns[None, :]] += s["scale"][a].double() * (t @ s["b"][a, columns, :rank].double().t())
    if case["act"] == "silu_mul":
        blocks = z.view(case["m"], -1, 32)
        z = (blocks[..., :16] * torch.sigmoid(blocks[..., :16]) * blocks[..., 16:]).reshape(case["m"], -1)
    return z


def _exact_tree(s, case):
    hq, hkv, d, page = (case[k] for k in ("hq", "hkv", "d", "page"))
    outs, lses, at = [], [], 0
    for j, (n, t) in enumerate(_lengths(case)):
        c = torch.arange(n, device="cuda")
        pages, inside = s["table"][j].long()[c // page], c % page
        i = torch.arange(t, device="cuda")[:, None]
        after = c[None, :] - (n - t)
        if case["masked"]:
            hidden = (after >= 0) & ((s["mask"][at:at + t] >> after.clamp(0, 63)) & 1 == 0)
        else:
            hidden = after > i
        out = torch.empty((t, hq, d), dtype=torch.float64, device="cuda")
        lse = torch.empty((t, hq), dtype=torch.float64, device="cuda")
        for h in range(hkv):
            k, v = s["k_cache"][pages, inside, h].double(), s["v_cache"][pages, inside, h].double()
            for u in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                score = s["q"][at:at + t, u].double() @ k.t() / math.sqrt(d)
                score[hidden] = -math.inf
                lse[:, u] = torch.logsumexp(score, -1)
                out[:, u] = torch.softmax(score, -1) @ v
        outs.append(out)
        lses.append(lse)
        at += t
    return torch.cat(outs), torch.cat(lses)
