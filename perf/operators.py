"""Performance cases of the operators around the cache: what a decoding program does besides forking and freeing.

  attend   decode attention over fork trees in a pool that keeps K and V in 4 bits (e2m1, a power-of-two scale per 32
           values): one request (a prompt and the threads forked off it) or many; `cand` > 0: the multi-candidate call
  prompt   attention of whole prompts over such a pool (causal), rows already there
  store    rows on their way into such a pool: thread created, prompt appended, rows read back, thread released
  rotate   rotary positions of q and k rows at given positions (`back`: transposed, as a gradient takes it)
  step     the same for one row of every listed thread, positions from the pool's books
  sample   a token for every row of logits, each row with its own temperature, top-k, top-p, min-p and random number

`own` false: elementary torch operations in 32 and 64 bits.  `own` true: the library's calls.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
D = 128
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- cases ----------------------------------------------------------------------------------------------
def _attend(name, hq, hkv, requests, prompt, kids, tail, cand=0, shape=1):
    c = {"kind": "attend", "hq": hq, "hkv": hkv, "requests": requests, "prompt_lo": prompt[0], "prompt_hi": prompt[1],
         "kids": kids, "tail_lo": tail[0], "tail_hi": tail[1], "cand": cand, "shape": shape}
    return dict(c, name=name) if name else c


def _rows(name, kind, hq, hkv, prompts, lo, hi, shape=1):
    c = {"kind": kind, "hq": hq, "hkv": hkv, "prompts": prompts, "lo": lo, "hi": hi, "shape": shape}
    return dict(c, name=name) if name else c


def _rotate(name, kind, hq, hkv, rows, dtype, dims, layout, scaling, far, fused, back):
    c = {"kind": kind, "hq": hq, "hkv": hkv, "rows": rows, "dtype": dtype, "dims": dims, "layout": layout, "scaling": scaling,
         "far": far, "fused": fused, "back": back}
    return dict(c, name=name) if name else c


def _sample(name, rows, vocab, dtype, cut):
    c = {"kind": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "cut": cut}
    return dict(c, name=name) if name else c


def listed():
    return [
        # interactive use: one layer's call for one user, five paragraphs in flight
        _attend("attend_one", 32, 8, 1, (300, 300), 5, (1, 40)),
        # one user with a long document, four threads on it
        _attend("attend_long", 32, 8, 1, (32001, 32001), 4, (20, 200)),
        # a server at an ordinary load, a kv head for every query head
        _attend("attend_64", 32, 32, 64, (256, 1024), 6, (8, 300)),
        # the largest: many requests with long prompts, grouped heads
        _attend("attend_256_long", 32, 8, 256, (2048, 4096), 4, (16, 512)),
        # verification of five candidates per thread
        _attend("attend_candidates", 32, 8, 24, (128, 1000), 8, (8, 300), cand=5),
        # long prompts arriving at a server
        _rows("prompt_long", "prompt", 32, 8, 5, 1000, 4500),
        # the rows of such prompts as they enter the cache
        _rows("store_prompts", "store", 32, 8, 6, 1024, 8192),
        # a decode step's query and key rows
        _rotate("rotate_step", "step", 32, 8, 48, "bf16", 128, "half", "none", 1200, False, False),
        # a prompt's rows out of one projection of q, k and v, contexts stretched by a ramp over the frequencies
        _rotate("rotate_prompt", "rotate", 32, 8, 16384, "bf16", 128, "half", "ramp", 131072, True, False),
        # the way back, in full precision, pairs side by side, half of the head
        _rotate("rotate_back", "rotate", 16, 16, 4099, "f32", 64, "pairs", "linear", 1 << 20, False, True),
        # one user's next token
        _sample("sample_one", 1, 32000, "bf16", "all"),
        # a batch's next tokens out of a large vocabulary
        _sample("sample_256", 256, 128000, "bf16", "all"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 8), (32, 32), (64, 8), (16, 4), (8, 8), (40, 8), (32, 2)]


def draw(rng):
    while True:
        kind = rng.choice(["attend"] * 5 + ["prompt"] * 2 + ["store", "rotate", "rotate", "step"] + ["sample"] * 4)
        shape = rng.randrange(1 << 20)
        if kind == "attend":
            hq, hkv = rng.choice(_HEADS)
            lo = _log(rng, 16, 30000)
            t = _log(rng, 1, 200)
            c = _attend(None, hq, hkv, _log(rng, 1, 256), (lo, int(lo * rng.uniform(1, 2.5))), rng.randint(1, 8),
                        (t, int(t * rng.uniform(1, 4))), rng.randint(1, 8) if rng.random() < 0.3 else 0, shape)
            m = max(1, c["cand"])
            most = c["requests"] * c["kids"] * (c["prompt_hi"] + c["tail_hi"])
            if most * hkv <= 1024 * 4608 * 8 and most * hq * m <= 1024 * 4608 * 32:
                return c
        elif kind == "prompt":
            hq, hkv = rng.choice([h for h in _HEADS if 16 % (h[0] // h[1]) == 0])
            lo = _log(rng, 16, 4000)
            c = _rows(None, kind, hq, hkv, _log(rng, 1, 32), lo, int(lo * rng.uniform(1, 3)), shape)
            if c["prompts"] * c["hi"] ** 2 * hq <= 5 * 4500 ** 2 * 32 and c["hi"] <= 8000:
                return c
        elif kind == "store":
            hq, hkv = rng.choice(_HEADS)
            lo = _log(rng, 1, 8000)
            c = _rows(None, kind, hq, hkv, _log(rng, 1, 32), lo, int(lo * rng.uniform(1, 3)), shape)
            if c["prompts"] * c["hi"] * hkv <= 6 * 8192 * 8:
                return c
        elif kind in ("rotate", "step"):
            hq, hkv = rng.choice(_HEADS)
            rows = _log(rng, 1, 20000) if kind == "rotate" else _log(rng, 1, 256)
            dtype = rng.choice(["bf16", "bf16", "f32"]) if kind == "rotate" else "bf16"
            c = _rotate(None, kind, hq, hkv, rows, dtype, rng.choice([128, 128, 64, 96, 32]), rng.choice(["half", "half", "pairs"]),
                        rng.choice(["none", "linear", "base", "ramp"]), _log(rng, 2048, 1 << 20) if kind == "rotate" else _log(rng, 16, 4096),
                        kind == "rotate" and rng.random() < 0.4, kind == "rotate" and rng.random() < 0.3)
            if work(c)["bytes"] <= 16384 * 40 * 512:
                return c
        else:
            c = _sample(None, _log(rng, 1, 512), _log(rng, 1000, 200000), rng.choice(["bf16", "bf16", "f32"]),
                        rng.choice(["all", "all", "none", "k", "p"]))
            if c["rows"] * c["vocab"] <= 256 * 128000:
                return c


def _lengths(case):
    """Prompt rows and own rows of the threads of every request, from the case alone."""
    rng = random.Random(case["shape"])
    if case["kind"] == "attend":
        return [(rng.randint(case["prompt_lo"], case["prompt_hi"]), [rng.randint(case["tail_lo"], case["tail_hi"]) for _ in range(case["kids"])])
                for _ in range(case["requests"])]
    return [(rng.randint(case["lo"], case["hi"]), []) for _ in range(case["prompts"])]


def work(case):
    """Bytes: each row held in 4 bits that a call attends to once (136 bytes per kv head: codes and scales of K and V), other inputs and
    outputs once.  Operations: two products per (query row, attended row); six per rotated pair; ten per logit."""
    kind = case["kind"]
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4), "flops": 10 * n}
    hq, hkv = case["hq"], case["hkv"]
    if kind in ("rotate", "step"):
        heads = case["rows"] * (hq + hkv)
        return {"bytes": 2 * heads * D * (2 if case["dtype"] == "bf16" else 4), "flops": 3 * heads * case["dims"]}
    lengths = _lengths(case)
    if kind == "attend":
        m = max(1, case["cand"])
        tokens = sum(p + sum(t) for p, t in lengths)
        threads = sum(len(t) for _, t in lengths)
        attended = sum(p + t for p, ts in lengths for t in ts) * m + threads * case["cand"] * (case["cand"] + 1) // 2
        return {"bytes": tokens * hkv * 136 + threads * m * hq * D * 4 + threads * case["cand"] * hkv * D * 4, "flops": 4 * D * hq * attended}
    tokens = sum(p for p, _ in lengths)
    if kind == "store":  # rows in, codes and scales out and in again, values out
        return {"bytes": tokens * hkv * (2 * D * 4 + 2 * 136), "flops": 8 * tokens * hkv * D}
    return {"bytes": tokens * (hkv * 136 + hq * D * 4), "flops": 4 * D * hq * sum(p * (p + 1) // 2 for p, _ in lengths)}


# ---- inputs ---------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _frequencies(case):
    """Per pair the angle of one position, as numbers (64 bits), and the factor on both sine and cosine."""
    r, base, factor = case["dims"], 10000.0, 8.0
    if case["scaling"] == "base":
        base *= factor ** (r / (r - 2))
    f = [base ** (-2.0 * i / r) for i in range(r // 2)]
    if case["scaling"] == "linear":
        f = [x / factor for x in f]
    if case["scaling"] == "ramp":
        keep = [min(max((8192 * x / (2 * math.pi) - 1.0) / 31.0, 0.0), 1.0) for x in f]
        f = [k * x + (1 - k) * x / factor for k, x in zip(keep, f)]
    return f, (0.1 * math.log(factor) + 1.0 if case["scaling"] == "ramp" else 1.0)


def _quantised(x):
    """Rows as the cache holds them: (codes, two to a byte, the even dim in the low half; exponents of the scales)."""
    y = x.float().reshape(*x.shape[:-1], 4, 32)
    f, k = torch.frexp(y.abs().amax(-1))
    e = torch.where(f <= 0.75, k - 3, k - 2).clamp(-120, 125)
    e = torch.where(f == 0, torch.zeros_like(e), e)
    y = torch.ldexp(y, -e[..., None]).clamp(-6, 6)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    code = torch.searchsorted(torch.tensor(_GRID, device=x.device), torch.round(a / step) * step)
    code = (code + 8 * (y < 0)).to(torch.uint8).reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), e.to(torch.int32)


def _cached(case, g):
    """K and V rows of every request, prompt first, then the threads' own rows; for every thread the rows on its path."""
    lengths = _lengths(case)
    first, paths = 0, []
    for p, tails in lengths:
        at = first + p
        for t in tails:
            paths.append((first, p, at, t))
            at += t
        if not tails:
            paths.append((first, p, at, 0))
        first = at
    k = torch.randn(first, case["hkv"], D, generator=g, device=DEV)
    k[..., 5::32] *= 3.0  # (a few loud channels)
    v = torch.randn(first, case["hkv"], D, generator=g, device=DEV)
    return lengths, paths, k.to(torch.bfloat16), v.to(torch.bfloat16)


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "sample":
        n, vocab = case["rows"], case["vocab"]
        x = torch.randn(n, vocab, generator=g, device=DEV) * 2.5
        x.add_(torch.randn(n, 64, generator=g, device=DEV).abs().mul_(5).repeat(1, -(-vocab // 64))[:, :vocab] * (torch.rand(n, vocab, generator=g, device=DEV) < 0.001))
        s["logits"] = x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        pick = lambda values: torch.tensor(values, device=DEV)[torch.randint(len(values), (n,), generator=g, device=DEV)]  # noqa: E731
        some = case["cut"]
        s["temperature"] = pick([0.0, 0.6, 0.8, 1.0, 1.0, 1.3])
        s["top_k"] = pick([0, 1, 20, 50, 500] if some in ("all", "k") else [0]).to(torch.int32)
        s["top_p"] = pick([1.0, 0.9, 0.95, 0.5] if some in ("all", "p") else [1.0])
        s["min_p"] = pick([0.0, 0.0, 0.05] if some == "all" else [0.0])
        s["u"] = torch.rand(n, generator=g, device=DEV)
        s["ids"] = (vocab - 3, vocab - 2, vocab - 1)  # the vocabulary's numbers of [Fork], [Child], [EOS]
        if own:
            import paper_2401_06761_amd as ap

            s["params"] = ap.apar_sample_rows(s["temperature"], s["top_k"], s["top_p"], s["min_p"])
            s["tokens"] = torch.empty(n, dtype=torch.int32, device=DEV)
            s["logprobs"] = torch.empty(n, device=DEV)
            s["workspace"] = torch.empty(ap.apar_sample_workspace_bytes(n, vocab), dtype=torch.uint8, device=DEV)
        return s
    hq, hkv = case["hq"], case["hkv"]
    if kind in ("rotate", "step"):
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        n = case["rows"]
        qkv = torch.randn(n, hq + 2 * hkv if case["fused"] else hq + hkv, D, generator=g, device=DEV).to(dtype)
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hkv]  # rows of one projection
        if not case["fused"]:
            s["q"], s["k"] = s["q"].contiguous(), s["k"].contiguous()
        s["positions"] = torch.randint(case["far"], (n,), generator=g, device=DEV, dtype=torch.int32)
        if kind == "step":
            s["positions"] = s["positions"].sort().values
        f, s["magnitude"] = _frequencies(case)
        s["theta"] = torch.tensor(f, dtype=torch.float64, device=DEV)
        s["q_out"] = torch.empty(n, hq, D, dtype=dtype, device=DEV)
        s["k_out"] = torch.empty(n, hkv, D, dtype=dtype, device=DEV)
        if own:
            import paper_2401_06761_amd as ap

            s["rotary"] = ap.Rotary(D, case["dims"], layout=case["layout"], base=10000.0, scaling=case["scaling"], factor=8.0, original_len=8192,
                                    low_turns=1.0, high_turns=32.0, magnitude=s["magnitude"])
            if kind == "step":  # one thread that grows, a child forked off it at every row's position
                at = s["positions"].tolist()
                s["pool"] = pool = ap.Pool(hq, hkv, D, "bf16_fp4kv", at[-1] // 16 + 2 + n, max_threads=n + 1, device=DEV)
                root, s["threads"] = ap.apar_thread_create(pool.handle), []
                rows = torch.zeros(max(1, at[-1]), hkv, D, dtype=dtype, device=DEV)
                have = 0
                for p in at:
                    ap.apar_append_kv(pool.handle, root, rows, rows, p - have)
                    have = p
                    s["threads"] += ap.apar_fork(pool.handle, root, 1)
                torch.cuda.synchronize()
        return s
    lengths, paths, k, v = _cached(case, g)
    if kind == "store":
        s["k"], s["v"] = k, v
    else:
        n = sum(p for p, _ in lengths) if kind == "prompt" else len(paths)
        m = max(1, case.get("cand", 0))
        s["q"] = (torch.randn(n, m, hq, D, generator=g, device=DEV) * 2.0).to(torch.bfloat16)
        if kind == "prompt":
            s["q"] = s["q"].reshape(n, hq, D)
        if m > 1 or case.get("cand", 0):
            s["cand_k"], s["cand_v"] = (torch.randn(n, m, hkv, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
            masks = []
            rng = random.Random(seed)
            for _ in range(n):
                rows = []
                for c in range(m):
                    rows.append((1 << c) | (rows[rng.randrange(c)] if c else 0))
                masks.append(rows)
            s["mask"] = torch.tensor(masks, dtype=torch.uint8, device=DEV)
    s["lens"] = [b + d for _, b, _, d in paths]
    if own:
        import paper_2401_06761_amd as ap

        blocks = sum(-(-p // 16) + sum(-(-t // 16) + 1 for t in ts) for p, ts in lengths) + 1
        s["pool"] = pool = ap.Pool(hq, hkv, D, "bf16_fp4kv", blocks, max_threads=1 << 30 if kind == "store" else len(paths) * 2 + 1, device=DEV)
        if kind == "store":
            s["k_out"], s["v_out"] = torch.empty_like(k), torch.empty_like(v)
            return s
        s["threads"], first = [], 0
        for p, tails in lengths:
            root = ap.apar_thread_create(pool.handle)
            ap.apar_append_kv(pool.handle, root, k[first:], v[first:], p)
            at = first + p
            for t, kid in zip(tails, ap.apar_fork(pool.handle, root, len(tails)) if tails else []):
                ap.apar_append_kv(pool.handle, kid, k[at:], v[at:], t)
                s["threads"].append(kid)
                at += t
            if tails:
                ap.apar_free_thread(pool.handle, root)
            else:
                s["threads"].append(root)
            first = at
        s["out"] = torch.empty_like(s["q"])
        torch.cuda.synchronize()
    elif kind != "store":
        s["k4"], s["v4"] = _quantised(k), _quantised(v)
        longest = max(s["lens"])
        at = torch.tensor(paths, device=DEV)[:, :, None]
        j = torch.arange(longest, device=DEV)[None]
        s["row_of"] = torch.where(j < at[:, 1], at[:, 0] + j, at[:, 2] + j - at[:, 1]).clamp(max=k.shape[0] - 1)
        s["len"] = torch.tensor(s["lens"], device=DEV)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------
def _values(packed):
    """[rows, heads, 128] in 32 bits of what the codes and exponents stand for."""
    codes, e = packed
    grid = torch.tensor(_GRID + tuple(-x for x in _GRID), device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 4, 32).int()
    return torch.ldexp(grid[c], e[..., None]).reshape(*codes.shape[:-1], D)


def _softmax_attention(q, k, v, seen):
    """q [T, M, hq, D], k, v [T, L, hkv, D], seen [T, M, L]: in 32 bits, heads side by side."""
    t, m, hq, _ = q.shape
    hkv = k.shape[2]
    q = q.float().reshape(t, m, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(t, hkv, -1, D)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)) * D ** -0.5
    s = s.reshape(t, hkv, -1, m, s.shape[-1]).masked_fill_(~seen[:, None, None], -math.inf)
    p = s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1)
    o = torch.matmul(p.reshape(t, hkv, -1, p.shape[-1]), v.permute(0, 2, 1, 3)).reshape(t, hkv, -1, m, D) / total[..., None]
    return o.permute(0, 3, 1, 2, 4).reshape(t, m, hq, D).to(torch.bfloat16)


def _plain_attend(s):
    k, v = _values(s["k4"])[s["row_of"]], _values(s["v4"])[s["row_of"]]
    t, longest = s["row_of"].shape
    m = s["q"].shape[1]
    seen = (torch.arange(longest, device=DEV) < s["len"][:, None])[:, None].expand(t, m, longest)
    if "mask" in s:
        k, v = torch.cat([k, s["cand_k"].float()], 1), torch.cat([v, s["cand_v"].float()], 1)
        seen = torch.cat([seen, (s["mask"][:, :, None].int() >> torch.arange(m, device=DEV)) & 1 > 0], 2)
    return _softmax_attention(s["q"], k, v, seen)


def _plain_prompt(s):
    k, v = _values(s["k4"])[s["row_of"]], _values(s["v4"])[s["row_of"]]
    longest = s["row_of"].shape[1]
    j = torch.arange(longest, device=DEV)
    here = j < s["len"][:, None]
    q = s["q"][s["row_of"]]  # (a prompt's queries are numbered as its rows)
    return _softmax_attention(q, k, v, (j[:, None] >= j).expand(len(here), longest, longest))[here]


def _plain_store(s):
    return [_values(_quantised(s[x])).to(torch.bfloat16) for x in ("k", "v")]


def _plain_rotated(x, s):
    case = s["case"]
    angle = s["positions"].double()[:, None] * s["theta"]
    cos, sin = ((f(angle) * s["magnitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    sin = -sin if case["back"] else sin
    r = case["dims"]
    y = x.float()
    a, b = (y[..., :r // 2], y[..., r // 2:r]) if case["layout"] == "half" else (y[..., 0:r:2], y[..., 1:r:2])
    c, d = a * cos - b * sin, b * cos + a * sin
    c = torch.cat([c, d], -1) if case["layout"] == "half" else torch.stack([c, d], -1).flatten(-2)
    return torch.cat([c, y[..., r:]], -1).to(x.dtype)


def _plain_sample(s):
    x = s["logits"].double()
    x, order = torch.sort(x, dim=-1, descending=True, stable=True)
    t = s["temperature"].double()[:, None]
    z = (x - x[:, :1]) / torch.where(t > 0, t, 1.0)
    rank = torch.arange(x.shape[1], device=x.device)
    k = torch.where(s["top_k"] > 0, s["top_k"], x.shape[1])[:, None]
    k = torch.where(t > 0, k, 1)
    w = torch.exp(z)
    p = s["top_p"].double()[:, None]
    among = w * (rank < k)
    before = torch.cumsum(among, -1) - among
    keep = (rank < k) & ((p >= 1) | (before < p * among.sum(-1, keepdim=True))) & (w >= s["min_p"].double()[:, None])
    keep[:, 0] = True
    kept = w * keep
    mass = kept.sum(-1, keepdim=True)
    at = (torch.cumsum(kept, -1) <= s["u"].double()[:, None] * mass).sum(-1, keepdim=True)
    at = torch.minimum(at, keep.sum(-1, keepdim=True) - 1)
    token = order.gather(1, at)[:, 0].int()
    logprob = (z.gather(1, at) - torch.log(mass))[:, 0].float()
    fork, child, eos = s["ids"]
    token = torch.where(token == fork, -1, torch.where(token == child, -2, torch.where(token == eos, -3, token)))
    return token, logprob


# ---- the library's calls --------------------------------------------------------------------------------
def _own_store(s):
    import paper_2401_06761_amd as ap

    pool, first, threads = s["pool"].handle, 0, []
    for n in s["lens"]:
        threads.append(ap.apar_thread_create(pool))
        ap.apar_append_kv(pool, threads[-1], s["k"][first:], s["v"][first:], n)
        first += n
    first = 0
    for t, n in zip(threads, s["lens"]):
        ap.apar_read_kv_rows(pool, t, 0, n, s["k_out"][first:], s["v_out"][first:])
        ap.apar_free_thread(pool, t)
        first += n
    return [s["k_out"], s["v_out"]]


def _own(s):
    import paper_2401_06761_amd as ap

    case = s["case"]
    kind = case["kind"]
    if kind == "store":
        return _own_store(s)
    if kind == "sample":
        ap.apar_sample_tokens(s["logits"], s["u"], s["tokens"], s["params"], token_ids=s["ids"], logprobs=s["logprobs"], workspace=s["workspace"])
        return s["tokens"], s["logprobs"]
    if kind == "rotate":
        ap.apar_rotate_rows(s["rotary"].handle, s["positions"], s["q"], s["k"], s["q_out"], s["k_out"], transposed=case["back"])
        return s["q_out"], s["k_out"]
    if kind == "step":
        ap.apar_rotate_threads(s["pool"].handle, s["rotary"].handle, s["threads"], s["q"], s["k"], s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    if kind == "prompt":
        ap.apar_prefill_attention(s["pool"].handle, s["q"], s["threads"], s["lens"], s["out"])
    elif case["cand"]:
        ap.apar_decode_attention_spec(s["pool"].handle, s["q"], s["cand_k"], s["cand_v"], s["mask"], case["cand"], s["threads"], s["out"])
    else:
        ap.apar_decode_attention(s["pool"].handle, s["q"], s["threads"], s["out"])
    return s["out"]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind in ("rotate", "step"):
        return _plain_rotated(state["q"], state), _plain_rotated(state["k"], state)
    return {"attend": _plain_attend, "prompt": _plain_prompt, "store": _plain_store, "sample": _plain_sample}[kind](state)


# ---- the same in 64 bits --------------------------------------------------------------------------------
def exact(case, seed):
    import numpy as np

    kind = case["kind"]

    def held(x):
        """The value nearest to each element on its group's grid, ties to the even code, by distance to all fifteen."""
        y = x.double().reshape(*x.shape[:-1], 4, 32)
        top = y.abs().amax(-1, keepdim=True)
        scale = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, 6.0) / 6.0)))
        scale = torch.where(top / scale > 6, scale * 2, torch.where(top / scale <= 3, scale / 2, scale))
        scale = torch.where(top > 0, scale, 1.0)
        best, away = torch.zeros_like(y), torch.full_like(y, math.inf)
        for i in (0, 2, 4, 6, 1, 3, 5, 7):  # (even codes first: an odd one has to be nearer)
            d = (y.abs() / scale - _GRID[i]).abs()
            best, away = torch.where(d < away, _GRID[i] * scale, best), torch.minimum(d, away)
        return (best * y.sign()).reshape(x.shape)

    if kind == "sample":
        s = prepare(case, seed)
        x = s["logits"].double().cpu().numpy()
        given = {n: s[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p", "u")}
        logprobs = np.empty(len(x))
        for r, row in enumerate(x):
            t = given["temperature"][r]
            row = np.sort(row)[::-1]
            if t <= 0:
                logprobs[r] = 0.0
                continue
            k = int(given["top_k"][r]) or len(row)
            w = np.exp((row[:k] - row[0]) / t)
            n = len(w) if given["top_p"][r] >= 1 else int(np.searchsorted(np.cumsum(w), given["top_p"][r] * w.sum(), side="left")) + 1
            w = w[:max(1, min(n, len(w)))]
            w = w[w >= min(given["min_p"][r], 1.0)]
            c = np.cumsum(w)
            at = min(int(np.searchsorted(c, given["u"][r] * c[-1], side="right")), len(w) - 1)
            logprobs[r] = np.log(w[at] / c[-1])
        return None, torch.from_numpy(logprobs)
    if kind in ("rotate", "step"):
        s = prepare(case, seed)
        theta, a = _frequencies(case)
        turn = s["positions"].double()[:, None] * torch.tensor(theta, dtype=torch.float64, device=DEV)
        turn = torch.polar(torch.full_like(turn, a), -turn if case["back"] else turn)[:, None]
        got = []
        for x in (s["q"], s["k"]):
            x, r = x.double(), case["dims"]
            if case["layout"] == "half":
                z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * turn
                y = torch.cat([z.real, z.imag, x[..., r:]], -1)
            else:
                z = torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous()) * turn
                y = torch.cat([torch.view_as_real(z).flatten(-2), x[..., r:]], -1)
            got.append(y)
        return tuple(got)
    if kind == "store":
        s = prepare(case, seed)
        return [held(s["k"]), held(s["v"])]
    # attention: the inputs again, from the seed, without what prepare() makes of them
    g = _generator(seed)
    lengths, paths, k, v = _cached(case, g)
    hq, hkv, m = case["hq"], case["hkv"], max(1, case.get("cand", 0))
    n = sum(p for p, _ in lengths) if kind == "prompt" else len(paths)
    s = prepare(case, seed)
    q = s["q"].double()
    k, v = held(k), held(v)
    out = torch.empty(n, hq, D, dtype=torch.float64, device=DEV) if kind == "prompt" else torch.empty(n, m, hq, D, dtype=torch.float64, device=DEV)
    row = 0
    for i, (first, p, at, t) in enumerate(paths):
        rows = torch.cat([torch.arange(first, first + p, device=DEV), torch.arange(at, at + t, device=DEV)])
        kk, vv = k[rows].transpose(0, 1), v[rows].transpose(0, 1)  # [hkv, L, D]
        length = p + t
        if kind == "prompt":
            for a in range(0, length, 1024):
                b = min(a + 1024, length)
                x = q[row + a:row + b].reshape(b - a, hkv, hq // hkv, D).permute(1, 2, 0, 3).reshape(hkv, -1, D)
                z = (x @ kk[:, :b].transpose(1, 2)).reshape(hkv, hq // hkv, b - a, b) / math.sqrt(D)
                z = z + torch.full((b - a, b), -math.inf, dtype=torch.float64, device=DEV).triu(a + 1)
                o = torch.softmax(z, -1).reshape(hkv, -1, b) @ vv[:, :b]
                out[row + a:row + b] = o.reshape(hkv, hq // hkv, b - a, D).permute(2, 0, 1, 3).reshape(b - a, hq, D)
            row += length
            continue
        for c in range(m):
            kc, vc = kk, vv
            if "mask" in s:
                bits = [j for j in range(m) if int(s["mask"][i, c]) >> j & 1]
                kc = torch.cat([kk, s["cand_k"][i, bits].double().transpose(0, 1)], 1)
                vc = torch.cat([vv, s["cand_v"][i, bits].double().transpose(0, 1)], 1)
            z = q[i, c].reshape(hkv, hq // hkv, D) @ kc.transpose(1, 2) / math.sqrt(D)
            out[i, c] = (torch.softmax(z, -1) @ vc).reshape(hq, D)
    return out
