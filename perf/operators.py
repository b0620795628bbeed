"""The operators of a serving iteration over paged key/value caches, as a user's program calls them on its own device
buffers: planning pages and slots for the requests, rotating and storing the new rows, attention of the new rows over the
pages, and drawing tokens from the logits.

`own` False: every operator in its plain form, elementary torch operations in 32 bits (64 where a border or an angle asks
for it).  `own` True: the package's entry points.  Heads and vocabularies are those of this repository's workloads (125M:
12 heads of 64; 1B: 16 of 128; 7B: 32 of 128; vocabularies 32000 and 32128) and the usual grouping of four query heads to a
key head.

Layout of a page, one head of it: keys in tiles of 16 positions x 32 dimensions, [position / 16][dim / 32][dim / 8 % 4]
[position % 16][dim % 8]; values in tiles of 32 positions x 16 dimensions, [position / 32][dim / 16][position / 4 % 4]
[dim % 16][position / 16 % 2][position % 4].
"""
import math

import torch

own = False

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
THETA = 10000.0


def listed():
    return [
        # one step of a small server: 16 requests, a verification of 5 rows each, next to no new pages
        dict(name="plan_16_verify", kind="plan", B=16, lo=100, hi=900, share_prompt=0.0, share_done=0.0, rows=5, chunk=0, page=64),
        # a large server's step: prompts in chunks among single rows, requests that end give their pages back
        dict(name="plan_1000_mixed", kind="plan", B=1000, lo=60, hi=20000, share_prompt=0.25, share_done=0.1, rows=3, chunk=600, page=32),
        # rows of a verification of 16 requests, four query heads to a key head
        dict(name="append_80_rows", kind="append", dtype="bf16", B=16, rows=5, lo=100, hi=5000, Hq=32, Hkv=8, hd=128, page=64),
        # prompts in large chunks at the 1B widths, page borders inside every chunk
        dict(name="append_8190_rows", kind="append", dtype="fp16", B=6, rows=1365, lo=1500, hi=9000, Hq=16, Hkv=16, hd=128, page=128),
        # the smallest call: one sequence, one new token, the 125M heads
        dict(name="attend_1_row_300", kind="attend", dtype="bf16", B=1, rows=1, big=0, big_rows=0, lo=300, hi=300, Hq=12, Hkv=12, hd=64, page=32),
        # a verification of 32 requests of all lengths, four query heads to a key head
        dict(name="attend_verify_32", kind="attend", dtype="bf16", B=32, rows=5, big=0, big_rows=0, lo=200, hi=8000, Hq=32, Hkv=8, hd=128, page=64),
        # long documents, one key head to each of the 7B model's query heads: the bytes of the cache alone
        dict(name="attend_long_60000", kind="attend", dtype="fp16", B=3, rows=9, big=0, big_rows=0, lo=23456, hi=59999, Hq=32, Hkv=32, hd=128, page=128),
        # a chunk of a long prompt over what is cached of it
        dict(name="attend_chunk_2048", kind="attend", dtype="bf16", B=1, rows=2048, big=0, big_rows=0, lo=8200, hi=8200, Hq=32, Hkv=8, hd=128, page=64),
        # chunks of two prompts among requests that generate
        dict(name="attend_mixed_24", kind="attend", dtype="fp16", B=24, rows=3, big=2, big_rows=509, lo=90, hi=5000, Hq=16, Hkv=16, hd=128, page=32),
        # one request's next token, all filters
        dict(name="sample_1_row", kind="sample", dtype="fp32", rows=1, vocab=32000, top_k=True, top_p=True, min_p=True),
        # the rows of 64 verifications, logits in half the bytes
        dict(name="sample_320_rows", kind="sample", dtype="bf16", rows=320, vocab=32000, top_k=True, top_p=True, min_p=False),
        # a large odd vocabulary, cut by probability alone: nearly every logit counts
        dict(name="sample_64_large_vocab", kind="sample", dtype="fp32", rows=64, vocab=128255, top_k=False, top_p=True, min_p=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "sample", "sample"])
    page = rng.choice([32, 64, 128, 256])
    if kind == "plan":
        return dict(kind=kind, B=_log(rng, 1, 1000), lo=_log(rng, 1, 200), hi=_log(rng, 300, 20000), share_prompt=rng.choice([0.0, 0.1, 0.25]),
                    share_done=rng.choice([0.0, 0.1]), rows=rng.randint(1, 16), chunk=_log(rng, 20, 600), page=page)
    Hq, Hkv, hd = rng.choice([(12, 12, 64), (16, 16, 128), (32, 32, 128), (32, 8, 128), (32, 4, 128), (24, 8, 64), (8, 1, 128)])
    dtype = rng.choice(["bf16", "fp16"])
    if kind == "append":
        B = _log(rng, 1, 64)
        rows = _log(rng, 1, max(2, 8000 // B))
        lo = rows + rng.randint(0, 300)
        return dict(kind=kind, dtype=dtype, B=B, rows=rows, lo=lo, hi=lo + _log(rng, 1, 4000), Hq=Hq, Hkv=Hkv, hd=hd, page=page)
    if kind == "attend":
        shape = rng.choice(["rows", "rows", "chunk", "mixed"])
        big = big_rows = 0
        if shape == "rows":
            B, rows = _log(rng, 1, 64), rng.choice([1, 1, rng.randint(2, 17)])
            lo = _log(rng, 1, 2000)
            hi = max(lo, min(_log(rng, 64, 59999), 5_000_000 // (B * Hkv)))
        elif shape == "chunk":
            B = rng.choice([1, 1, 2, 3])
            rows = _log(rng, 18, 2000 // B)
            lo = rows if rng.random() < 0.3 else _log(rng, rows, 8000)
            hi = max(lo, min(_log(rng, 500, 8000), 500_000_000 // (B * rows * Hq)))
        else:
            B, rows, big, big_rows = rng.randint(3, 24), rng.randint(1, 9), rng.randint(1, 2), _log(rng, 18, 500)
            lo = _log(rng, 1, 700)
            hi = max(lo, min(_log(rng, 700, 5000), 900_000_000 // (B * big_rows * Hq)))
        return dict(kind=kind, dtype=dtype, B=B, rows=rows, big=big, big_rows=big_rows, lo=lo, hi=hi, Hq=Hq, Hkv=Hkv, hd=hd, page=page)
    vocab = rng.choice([1024, 32000, 32128, rng.randint(500, 50000), rng.randint(50001, 128255)])
    return dict(kind=kind, dtype=rng.choice(["fp32", "bf16", "fp16"]), rows=_log(rng, 1, min(320, 9_000_000 // vocab)), vocab=vocab,
                top_k=rng.random() < 0.6, top_p=rng.random() < 0.6, min_p=rng.random() < 0.4)


# ---- the requests of a case: the same for every seed, so that its work is known -------------------------------------
def _lengths(c):
    """Lengths spread evenly over the logarithm of lo .. hi."""
    B, lo, hi = c["B"], c["lo"], c["hi"]
    return [int(round(lo * (hi / lo) ** (i / max(1, B - 1)))) for i in range(B)]


def _requests(c):
    """(cached, fresh) of each request; the order is a fixed shuffle of the lengths."""
    B = c["B"]
    step = next(s for s in range(max(1, int(B * 0.618)), B + 2) if math.gcd(s, B) == 1)
    lens = _lengths(c)
    lens = [lens[i * step % B] for i in range(B)]
    out = []
    for i, n in enumerate(lens):
        if c["kind"] == "plan":
            if (i * 7919 % 1000) < 1000 * c["share_done"]:
                out.append((0, 0))
            elif (i * 104729 % 1000) < 1000 * c["share_prompt"]:
                out.append((n // 2, c["chunk"] - i % 13))
            else:
                out.append((n, c["rows"]))
        elif c["kind"] == "append":
            out.append((n - min(n, c["rows"]), min(n, c["rows"])))
        else:
            r = min(n, c["big_rows"] if i >= B - c["big"] else c["rows"])
            out.append((n - r, r))
    return out


def _pages(n, page):
    return -(-n // page)


def work(c):
    if c["kind"] == "sample":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * (4 if c["dtype"] == "fp32" else 2) + c["rows"] * 28, "flops": 4 * n}
    req = _requests(c)
    rows = sum(f for _, f in req)
    if c["kind"] == "plan":
        return {"bytes": 4 * (3 * c["B"] + 3 * c["B"] + 2 * rows) + 8 * sum(_pages(f, c["page"]) for _, f in req), "flops": rows}
    if c["kind"] == "append":
        return {"bytes": 2 * rows * c["hd"] * (2 * c["Hq"] + 4 * c["Hkv"]) + 8 * rows, "flops": 3 * rows * c["hd"] * (c["Hq"] + c["Hkv"])}
    seen = sum(f * a + f * (f + 1) // 2 for a, f in req)
    kv = sum(a + f for a, f in req)
    return {"bytes": 2 * c["hd"] * (2 * kv * c["Hkv"] + 2 * rows * c["Hq"]), "flops": 4 * c["hd"] * c["Hq"] * seen}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _ints(values, dev):
    return torch.tensor(values, dtype=torch.int32, device=dev)


def _offsets(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def prepare(c, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    if c["kind"] == "sample":
        n, V = c["rows"], c["vocab"]
        # a trained model's logits: a wide bulk and a few tokens far above it
        x = torch.randn(n, V, generator=g, device=dev) * 2.0
        at = torch.randint(0, V, (n, 24), generator=g, device=dev)
        x.scatter_add_(1, at, torch.rand(n, 24, generator=g, device=dev) * 9.0)
        one = lambda: torch.rand(n, generator=g, device=dev)  # noqa: E731
        return dict(c, logits=x.to(DT[c["dtype"]]), temperature=0.4 + one(), uniform=one(),
                    top_k_of=(1 + one() * 199).int() if c["top_k"] else None,
                    top_p_of=0.6 + 0.39 * one() if c["top_p"] else None, min_p_of=0.1 * one() if c["min_p"] else None,
                    token=torch.empty(n, dtype=torch.int32, device=dev), logprob=torch.empty(n, device=dev),
                    kept=torch.empty(n, dtype=torch.int32, device=dev))
    req, ps, B = _requests(c), c["page"], c["B"]
    rows = sum(f for _, f in req)
    shuffled = lambda n: torch.randperm(n, generator=g, device=dev).int()  # noqa: E731
    if c["kind"] == "plan":
        lens = _lengths(c)
        held = [_pages(a, ps) if a + f else _pages(lens[i], ps) for i, (a, f) in enumerate(req)]
        most = max(max(held), max(_pages(a + f, ps) for a, f in req)) + 3
        spare = sum(max(0, _pages(a + f, ps) - h) for (a, f), h in zip(req, held)) + 17
        n_pages = sum(held) + spare
        order = shuffled(n_pages)
        table = torch.full((B, most), -1, dtype=torch.int32, device=dev)
        start = torch.tensor(_offsets(held)[:-1], device=dev)
        at = torch.arange(most, device=dev)
        has = at[None] < _ints(held, dev)[:, None]
        table = torch.where(has, order[(start[:, None] + at[None]).clamp(max=n_pages - 1)], table)
        free = torch.full((n_pages,), -1, dtype=torch.int32, device=dev)
        free[:spare] = order[sum(held):]
        cap = rows + 9                                  # rows of the program's buffers: a few behind the last request's
        return dict(c, n_pages=n_pages, max_blocks=most, cap=cap, cached=_ints([a for a, _ in req], dev), fresh=_ints([f for _, f in req], dev),
                    held=_ints(held, dev), n_free=_ints([spare], dev), table=table, free=free,
                    held_out=torch.empty(B, dtype=torch.int32, device=dev), n_free_out=torch.empty(1, dtype=torch.int32, device=dev),
                    row_start=torch.empty(B + 1, dtype=torch.int32, device=dev), seq_len=torch.empty(B, dtype=torch.int32, device=dev),
                    position=torch.empty(cap, dtype=torch.int32, device=dev), slot=torch.empty(cap, dtype=torch.int32, device=dev))
    Hq, Hkv, hd, dt = c["Hq"], c["Hkv"], c["hd"], DT[c["dtype"]]
    held = [_pages(a + f, ps) for a, f in req]
    most = max(held) + 1
    n_pages = sum(held) + 2
    order = shuffled(n_pages)
    at = torch.arange(most, device=dev)
    start = torch.tensor(_offsets(held)[:-1], device=dev)
    table = torch.where(at[None] < _ints(held, dev)[:, None], order[(start[:, None] + at[None]).clamp(max=n_pages - 1)],
                        torch.full((B, most), -1, dtype=torch.int32, device=dev))
    normal = lambda *s: torch.randn(*s, generator=g, device=dev, dtype=dt)  # noqa: E731
    s = dict(c, n_pages=n_pages, max_blocks=most, table=table,
             k_pages=normal(n_pages, Hkv, ps // 16, hd // 32, 4, 16, 8), v_pages=normal(n_pages, Hkv, ps // 32, hd // 16, 4, 16, 2, 4))
    row_start = _offsets([f for _, f in req])
    if c["kind"] == "append":
        position = torch.cat([torch.arange(a, a + f, device=dev) for a, f in req])
        seq = torch.repeat_interleave(torch.arange(B, device=dev), torch.tensor([f for _, f in req], device=dev))
        slot = table[seq, position // ps].long() * ps + position % ps
        qkv = normal(rows, (Hq + 2 * Hkv) * hd)         # one projection's output: q, k and v are slices of its rows
        return dict(s, rows_in=rows, qkv=qkv, position=position.int(), slot=slot.int(), q_out=torch.empty(rows, Hq * hd, dtype=dt, device=dev))
    cap = rows + 3                                      # rows of the program's buffers: a few behind the last request's
    return dict(s, cap=cap, max_fresh=max(f for _, f in req), q=normal(cap, Hq * hd), out=torch.zeros(cap, Hq * hd, dtype=dt, device=dev),
                row_start=_ints(row_start, dev), seq_len=_ints([a + f for a, f in req], dev))


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _plain_plan(s):
    B, ps, most, n_pages, cap = s["B"], s["page"], s["max_blocks"], s["n_pages"], s["cap"]
    cached, fresh, held, table, free = s["cached"].long(), s["fresh"].long(), s["held"].long(), s["table"], s["free"]
    n_free = s["n_free"].long()
    need = (cached + fresh + ps - 1) // ps
    fits = need <= most
    ask, drop = torch.where(fits, (need - held).clamp(min=0), 0), (held - need).clamp(min=0)
    ask_to, drop_to = ask.cumsum(0), drop.cumsum(0)
    avail = n_free + drop_to[-1:]
    ok = ((ask == 0) | (ask_to <= avail)) & fits
    grant = torch.where(ok, ask, 0)
    at = torch.arange(most, device=table.device)[None]
    # pages given back go behind the free ones, in the order of the requests
    gives = (at >= need[:, None]) & (at < held[:, None])
    to = torch.where(gives, n_free + (drop_to - drop)[:, None] + at - need[:, None], n_pages)
    stack = torch.cat([free, free[:1]]).scatter(0, to.reshape(-1), table.reshape(-1))[:n_pages]
    # pages granted come from the end of the stack
    takes = (at >= held[:, None]) & (at < (held + grant)[:, None])
    frm = torch.where(takes, avail - 1 - (ask_to - ask)[:, None] - (at - held[:, None]), 0)
    table = torch.where(takes, stack[frm], table)
    row_start = torch.cat([torch.zeros_like(fresh[:1]), fresh.cumsum(0)])
    t = torch.arange(cap, device=table.device)
    b = torch.searchsorted(row_start[1:].contiguous(), t, right=True)
    live = b < B
    b = b.clamp(max=B - 1)
    live &= ok[b]
    pos = cached[b] + t - row_start[b]
    page = table[b, torch.where(live, pos // ps, 0)].long()
    i32 = lambda v: v.int()  # noqa: E731
    return dict(table=table, free=stack, held=i32(torch.where(ok, torch.where(ask > 0, held + grant, need), held)),
                n_free=i32(avail - grant.sum()), row_start=i32(row_start), seq_len=i32(torch.where(ok, cached + fresh, 0)),
                position=i32(torch.where(live, pos, -1)), slot=i32(torch.where(live, page * ps + pos % ps, -1)))


def _rotate(x, position, hd):
    """Pairs (i, i + hd / 2) of x [rows, heads, hd] turned by position * theta^(-2i / hd), angles in 64 bits."""
    i = torch.arange(hd // 2, device=x.device, dtype=torch.float64)
    angle = position.double()[:, None] * THETA ** (-2.0 * i / hd)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x[..., : hd // 2], x[..., hd // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _split(s):
    Hq, Hkv, hd, n = s["Hq"], s["Hkv"], s["hd"], s["rows_in"]
    q, k, v = s["qkv"].split([Hq * hd, Hkv * hd, Hkv * hd], 1)
    return q.view(n, Hq, hd), k.view(n, Hkv, hd), v.view(n, Hkv, hd)


def _plain_append(s):
    Hkv, hd, ps, n = s["Hkv"], s["hd"], s["page"], s["rows_in"]
    q, k, v = _split(s)
    dt = q.dtype
    page, at = s["slot"].long() // ps, s["slot"].long() % ps
    kr = _rotate(k.float(), s["position"], hd).to(dt)
    s["k_pages"][page, :, at // 16, :, :, at % 16] = kr.view(n, Hkv, hd // 32, 4, 8)
    s["v_pages"][page, :, at // 32, :, at // 4 % 4, :, at // 16 % 2, at % 4] = v.reshape(n, Hkv, hd // 16, 16)
    return dict(k=s["k_pages"], v=s["v_pages"], q=_rotate(q.float(), s["position"], hd).to(dt).view(n, -1))


def _logical(pages_of, value):
    """Pages as they are addressed, [.., blocks, heads, tiles ...] -> [B, heads, positions, hd]."""
    if not value:
        B, m, H, t, e, f, p, j = pages_of.shape
        return pages_of.permute(0, 2, 1, 3, 6, 4, 5, 7).reshape(B, H, m * t * p, e * f * j)
    B, m, H, t, e, g, d, h, i = pages_of.shape
    return pages_of.permute(0, 2, 1, 3, 7, 5, 8, 4, 6).reshape(B, H, m * t * h * g * i, e * d)


def _plain_attend(s):
    B, Hq, Hkv, hd, nf, cap = s["B"], s["Hq"], s["Hkv"], s["hd"], s["max_fresh"], s["cap"]
    G = Hq // Hkv
    dev = s["q"].device
    row_start, seq_len, table = s["row_start"].long(), s["seq_len"].long(), s["table"].long().clamp(min=0)
    K = _logical(s["k_pages"][table], False).float()
    V = _logical(s["v_pages"][table], True).float()
    L = K.shape[2]
    fresh = row_start[1:] - row_start[:-1]
    r = torch.arange(nf, device=dev)
    row = (row_start[:-1, None] + r[None]).clamp(max=cap - 1)
    q = s["q"].view(cap, Hkv, G, hd)[row].float()                            # [B, nf, Hkv, G, hd]
    q = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, nf * G, hd) * (1.0 / math.sqrt(hd))
    x = torch.matmul(q, K.transpose(2, 3).contiguous())                      # [B, Hkv, nf * G, L]
    pos = (seq_len - fresh)[:, None] + r[None]
    sees = torch.arange(L, device=dev)[None, None] <= torch.minimum(pos, seq_len[:, None] - 1)[:, :, None]
    x = x.view(B, Hkv, nf, G, L).masked_fill_(~sees[:, None, :, None], -math.inf).view(B, Hkv, nf * G, L)
    x = x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    o = torch.matmul(x, V) / x.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.view(B, Hkv, nf, G, hd).permute(0, 2, 1, 3, 4).reshape(B, nf, Hq * hd).to(s["q"].dtype)
    t = torch.arange(cap, device=dev)
    b = torch.searchsorted(row_start[1:].contiguous(), t, right=True)
    live = b < B
    b = b.clamp(max=B - 1)
    return torch.where(live[:, None], o[b, (t - row_start[b]).clamp(0, nf - 1)], s["out"])


def _plain_sample(s):
    n, V = s["rows"], s["vocab"]
    x = s["logits"].double()
    x = torch.where(x.isnan(), -math.inf, x)
    T = s["temperature"].double()[:, None]
    xs, idx = x.sort(dim=1, descending=True, stable=True)
    w = torch.where(xs == xs[:, :1], 0.0, (xs - xs[:, :1]) / T).exp()
    rank = torch.arange(V, device=x.device)[None]
    if s["top_k_of"] is not None:
        k = s["top_k_of"].long()[:, None]
        w = torch.where((rank < k) | (k <= 0), w, 0.0)
    keep = w > 0
    if s["top_p_of"] is not None:
        p = s["top_p_of"].double()[:, None]
        to = w.cumsum(1)
        before = torch.cat([torch.zeros_like(to[:, :1]), to[:, :-1]], 1)
        keep &= (before < p * to[:, -1:]) | (p >= 1) | (rank == 0)
    if s["min_p_of"] is not None:
        keep &= w >= s["min_p_of"].double()[:, None].clamp(max=1.0)
    kw = torch.zeros_like(w).scatter(1, idx, torch.where(keep, w, 0.0))
    to = kw.cumsum(1)
    Z = to[:, -1:]
    token = torch.searchsorted(to, s["uniform"].double()[:, None] * Z, right=True).clamp(max=V - 1)
    return dict(token=token[:, 0].int(), logprob=(kw.gather(1, token) / Z).log()[:, 0].float(), kept=keep.sum(1).int())


# ---- the package's entry points -------------------------------------------------------------------------------------
def _bind(s):
    """The program's buffers as the entry points take them, and the workspace they ask for."""
    import paper_2407_19947_amd as pkg
    code = {"fp32": pkg.DTYPE_FP32, "bf16": pkg.DTYPE_BF16, "fp16": pkg.DTYPE_FP16}
    at = lambda name: s[name].data_ptr() if s[name] is not None else None  # noqa: E731
    if s["kind"] == "plan":
        p = pkg.StairsPagePlan(n_seqs=s["B"], max_blocks=s["max_blocks"], n_pages=s["n_pages"], page_size=s["page"], max_rows=s["cap"],
                               cached=at("cached"), fresh=at("fresh"), held=at("held"), n_free=at("n_free"), block_table=at("table"),
                               free_pages=at("free"), held_out=at("held_out"), n_free_out=at("n_free_out"), row_start=at("row_start"),
                               seq_len=at("seq_len"), position=at("position"), slot=at("slot"))
        return lambda stream: pkg.stairs_paged_plan(p, stream)
    if s["kind"] == "sample":
        a = pkg.StairsSampling(dtype=code[s["dtype"]], rows=s["rows"], vocab=s["vocab"], ld=s["vocab"], logits=at("logits"),
                               temperature=at("temperature"), top_k=at("top_k_of"), top_p=at("top_p_of"), min_p=at("min_p_of"),
                               uniform=at("uniform"), token=at("token"), logprob=at("logprob"), kept=at("kept"))
        s["work"] = torch.zeros(pkg.stairs_sample_workspace(a), dtype=torch.uint8, device=s["logits"].device)
        a.workspace, a.workspace_bytes = s["work"].data_ptr(), s["work"].numel()
        return lambda stream: pkg.stairs_sample_device(a, stream)
    cache = pkg.StairsPagedCache(k=at("k_pages"), v=at("v_pages"), dtype=code[s["dtype"]], n_pages=s["n_pages"], page_size=s["page"],
                                 n_kv_heads=s["Hkv"], head_dim=s["hd"])
    if s["kind"] == "append":
        q, k, v = _split(s)
        ld = s["qkv"].stride(0)
        r = pkg.StairsPagedRows(rows=s["rows_in"], n_heads=s["Hq"], q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), q_out=at("q_out"),
                                q_stride=ld, k_stride=ld, v_stride=ld, q_out_stride=s["q_out"].stride(0),
                                position=at("position"), slot=at("slot"), rope_theta=THETA)
        return lambda stream: pkg.stairs_paged_append(cache, r, stream)
    a = pkg.StairsPagedAttention(n_seqs=s["B"], max_blocks=s["max_blocks"], rows=s["cap"], n_heads=s["Hq"], max_fresh=s["max_fresh"],
                                 q=at("q"), out=at("out"), q_stride=s["q"].stride(0), out_stride=s["out"].stride(0),
                                 block_table=at("table"), row_start=at("row_start"), seq_len=at("seq_len"), scale=0.0)
    s["work"] = torch.zeros(pkg.stairs_paged_attention_workspace(cache, a), dtype=torch.uint8, device=s["q"].device)
    a.workspace, a.workspace_bytes = s["work"].data_ptr(), s["work"].numel()
    return lambda stream: pkg.stairs_paged_attention(cache, a, stream)


def _own(s):
    call = s.get("call")
    if call is None:
        call = s["call"] = _bind(s)
    call(torch.cuda.current_stream().cuda_stream)
    if s["kind"] == "plan":
        return dict(table=s["table"], free=s["free"], held=s["held_out"], n_free=s["n_free_out"], row_start=s["row_start"],
                    seq_len=s["seq_len"], position=s["position"], slot=s["slot"])
    if s["kind"] == "append":
        return dict(k=s["k_pages"], v=s["v_pages"], q=s["q_out"])
    if s["kind"] == "attend":
        return s["out"]
    return dict(token=s["token"], logprob=s["logprob"], kept=s["kept"])


def run(state):
    if own:
        return _own(state)
    return {"plan": _plain_plan, "append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}[state["kind"]](state)


# ---- definitions in 64 bits --------------------------------------------------------------------------------------
def _exact_pages(raw, value):
    """The pages of one head order as [pages, heads, positions, hd] in 64 bits, by the address of every element."""
    n, H = raw.shape[:2]
    flat = raw.reshape(n, H, -1)
    hd = raw.shape[3] * (16 if value else 32)
    ps = flat.shape[2] // hd
    p, e = torch.meshgrid(torch.arange(ps, device=raw.device), torch.arange(hd, device=raw.device), indexing="ij")
    if value:
        at = (((p // 32) * (hd // 16) + e // 16) * 64 + e % 16 + 16 * (p % 16 // 4)) * 8 + p % 4 + 4 * (p % 32 // 16)
    else:
        at = (((p // 16) * (hd // 32) + e // 32) * 64 + p % 16 + 16 * (e % 32 // 8)) * 8 + e % 8
    return flat, at


def exact(c, seed):
    if c["kind"] == "plan":
        return None                                     # whole numbers only
    s = prepare(c, seed)
    if c["kind"] == "sample":
        lp = []
        x = s["logits"].double().cpu()
        for r in range(c["rows"]):
            v = x[r]
            w = ((v - v.max()) / float(s["temperature"][r])).exp()
            idx = torch.argsort(v, descending=True, stable=True)
            if s["top_k_of"] is not None:
                idx = idx[: max(1, int(s["top_k_of"][r]))]
            if s["top_p_of"] is not None:
                total = math.fsum(w[idx].tolist())
                to = torch.cumsum(w[idx], 0)
                idx = idx[: 1 + int((to[:-1] < float(s["top_p_of"][r]) * total).sum())]
            if s["min_p_of"] is not None:
                idx = idx[w[idx] >= float(s["min_p_of"][r])]
            idx = torch.sort(idx).values
            to = torch.cumsum(w[idx], 0)
            t = idx[min(int((to <= float(s["uniform"][r]) * float(to[-1])).sum()), len(idx) - 1)]
            lp.append(float(torch.log(w[t] / to[-1])))
        return dict(token=None, logprob=torch.tensor(lp, dtype=torch.float64), kept=None)
    hd, ps, Hq, Hkv = c["hd"], c["page"], c["Hq"], c["Hkv"]
    fk, ak = _exact_pages(s["k_pages"], False)
    fv, av = _exact_pages(s["v_pages"], True)
    if c["kind"] == "append":
        q, k, v = (t.double() for t in _split(s))
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device=q.device),
                           s["position"].double()[:, None] / THETA ** (torch.arange(hd // 2, device=q.device, dtype=torch.float64) * (2.0 / hd)))[:, None]
        turned = lambda x: torch.view_as_real(torch.complex(x[..., : hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * turn).transpose(-1, -2).reshape(x.shape)  # noqa: E731
        fk, fv = fk.double(), fv.double()
        page, p = s["slot"].long() // ps, s["slot"].long() % ps
        head = torch.arange(Hkv, device=q.device)
        fk[page[:, None, None], head[None, :, None], ak[p][:, None]] = turned(k)
        fv[page[:, None, None], head[None, :, None], av[p][:, None]] = v
        return dict(k=fk.view(s["k_pages"].shape), v=fv.view(s["v_pages"].shape), q=turned(q).reshape(len(p), -1))
    out = s["out"].double()
    for b, (a, f) in enumerate(_requests(c)):
        n = a + f
        ids = s["table"][b, : _pages(n, ps)].long()
        r0 = int(s["row_start"][b])
        visible = torch.arange(n, device=out.device)[None] <= a + torch.arange(f, device=out.device)[:, None]
        for h in range(Hkv):
            K = fk[ids, h][:, ak].reshape(-1, hd)[:n].double()
            V = fv[ids, h][:, av].reshape(-1, hd)[:n].double()
            for gq in range(Hq // Hkv):
                col = (h * (Hq // Hkv) + gq) * hd
                x = s["q"][r0: r0 + f, col: col + hd].double() @ K.T.contiguous() / math.sqrt(hd)
                out[r0: r0 + f, col: col + hd] = torch.softmax(torch.where(visible, x, -math.inf), 1) @ V
    return out
