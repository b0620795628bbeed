"""What the tests of the operators on device buffers share: plain implementations in 64 bits (numpy, a loop over requests and
rows), page addressing by its formula, and the calls with torch owning the buffers."""
import math

import numpy as np

import paper_2407_19947_amd as pkg

HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
CODE = {"fp32": pkg.DTYPE_FP32, "bf16": pkg.DTYPE_BF16, "fp16": pkg.DTYPE_FP16}


SMALLEST = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25}       # half of the smallest step: what rounding costs next to 0


def check_close(got, want, tol, what=""):
    """|got - want| <= tol everywhere; else the worst place is said."""
    off = np.abs(got - want)
    bad = ~(off <= tol)
    if bad.any():
        at = np.unravel_index(np.argmax(np.where(bad, off / np.maximum(tol, 1e-300), 0)), bad.shape)
        raise AssertionError(f"{what} {int(bad.sum())} of {bad.size} off, worst at {tuple(map(int, at))}: {got[at]!r} for {want[at]!r}, allowed {tol[at]!r}")


def torch_type(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


# ---- pages -------------------------------------------------------------------------------------------------------------
def key_at(p, e, hd):
    return (((p // 16) * (hd // 32) + e // 32) * 64 + p % 16 + 16 * (e % 32 // 8)) * 8 + e % 8


def value_at(p, e, hd):
    return (((p // 32) * (hd // 16) + e // 16) * 64 + e % 16 + 16 * (p % 16 // 4)) * 8 + p % 4 + 4 * (p % 32 // 16)


def pages_to_rows(raw, hd, at):
    """[pages, heads, page_size * hd] -> [pages, heads, page_size, hd]"""
    ps = raw.shape[2] // hd
    p, e = np.meshgrid(np.arange(ps), np.arange(hd), indexing="ij")
    return raw[:, :, at(p, e, hd)]


def rows_to_pages(rows, at):
    n, h, ps, hd = rows.shape
    p, e = np.meshgrid(np.arange(ps), np.arange(hd), indexing="ij")
    raw = np.empty((n, h, ps * hd), rows.dtype)
    raw[:, :, at(p, e, hd)] = rows
    return raw


def plan_reference(cached, fresh, held, table, free, n_free, page, max_rows):
    """The plan one request after the other; table and free are changed."""
    n_pages, most = len(free), table.shape[1]
    cached, fresh = [max(int(c), 0) for c in cached], [max(int(f), 0) for f in fresh]
    held = [min(max(int(h), 0), most) for h in held]
    need = [-(-(c + f) // page) for c, f in zip(cached, fresh)]
    for b, n in enumerate(need):
        if n <= most:
            for j in range(n, held[b]):
                free[n_free] = table[b, j]
                n_free += 1
    budget, asked = n_free, 0
    held_out, seq_len, position, slot, start = list(held), [], [], [], [0]
    for b, n in enumerate(need):
        ok = n <= most
        if ok and n > held[b]:
            asked += n - held[b]
            ok = asked <= budget
            if ok:
                for j in range(held[b], n):
                    n_free -= 1
                    table[b, j] = free[n_free]
        if ok:
            held_out[b] = n
        seq_len.append(cached[b] + fresh[b] if ok else 0)
        for i in range(fresh[b]):
            p = cached[b] + i
            position.append(p if ok else -1)
            slot.append(int(table[b, p // page]) * page + p % page if ok and 0 <= table[b, p // page] < n_pages else -1)
        start.append(start[-1] + fresh[b])
    pad = lambda v: (v + [-1] * max_rows)[:max_rows]  # noqa: E731
    return dict(held=held_out, n_free=n_free, seq_len=seq_len, row_start=start, position=pad(position), slot=pad(slot))


# ---- attention -----------------------------------------------------------------------------------------------------
def attention_reference(q, K, V, table, row_start, seq_len, scale, half, smallest=2.0 ** -25):
    """q [rows, Hq, hd], K and V [pages, Hkv, page_size, hd] in float64 -> (out, allowed error; rows nobody has: NaN, 0).

    The error allowed, element by element, with h the half step of the type and A = sum_j p_j |v_j|: the output's rounding h |o| (2^-25
    next to 0 in half);
    the probabilities' rounding h A; scores added in float, an error of (hd + 2) 2^-24 sum |q k| scale + the exponent's 2^-22 |x|, in
    every probability and in their sum, hence twice; sums over the keys in float, (L + 64) 2^-24 A, twice (numerator, denominator)."""
    rows, Hq, hd = q.shape
    n_pages, Hkv, ps, _ = K.shape
    out, tol = np.full((rows, Hq, hd), np.nan), np.zeros((rows, Hq, hd))
    for b in range(len(seq_len)):
        f, n = row_start[b + 1] - row_start[b], int(seq_len[b])
        blocks = np.array([table[b, j] if j < table.shape[1] else -1 for j in range(-(-n // ps))], int)
        there = np.repeat((blocks >= 0) & (blocks < n_pages), ps)[:n]
        at = np.where((blocks >= 0) & (blocks < n_pages), blocks, 0)
        for h in range(Hq):
            k = K[at, h // (Hq // Hkv)].reshape(-1, hd)[:n]
            v = V[at, h // (Hq // Hkv)].reshape(-1, hd)[:n]
            for i in range(f):
                t = row_start[b] + i
                sees = there & (np.arange(n) <= n - f + i)
                if not sees.any():
                    out[t, h] = 0
                    continue
                ks, vs = k[sees], v[sees]
                x = ks @ q[t, h] * scale
                with np.errstate(invalid="ignore", over="ignore"):
                    p = np.exp(x - x.max())
                    p /= p.sum()
                    out[t, h] = p @ vs
                    A = p @ np.abs(vs)
                    d = 2 * ((hd + 2) * 2.0 ** -24 * (np.abs(ks) @ np.abs(q[t, h])).max() * scale + 2.0 ** -22 * (x.max() - x).max()) \
                        + 2 * (len(x) + 64) * 2.0 ** -24
                    tol[t, h] = half * np.abs(out[t, h]) + A * (half + d) + smallest
    return out, tol


class Attend:
    """Sequences over a random pool: lens (new rows included), fresh rows each."""

    def __init__(self, dtype, lens, fresh, Hq, Hkv, hd, page, seed=0, spare_rows=2, q_scale=1.0, extra_blocks=1):
        import torch
        self.dt, self.dtype, self.hd, self.page, self.Hq, self.Hkv = torch_type(dtype), dtype, hd, page, Hq, Hkv
        self.lens, self.fresh = list(lens), list(fresh)
        rng = np.random.default_rng([seed, len(lens), sum(lens), Hq, hd, page])
        held = [-(-n // page) for n in lens]
        self.n_pages = sum(held) + 2
        order = rng.permutation(self.n_pages)
        self.max_blocks = max(held + [1]) + extra_blocks
        self.table = np.full((max(len(lens), 1), self.max_blocks), -1, np.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.row_start = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
        self.rows = int(self.row_start[-1]) + spare_rows
        g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
        normal = lambda *s: torch.randn(*s, generator=g).to(self.dt)  # noqa: E731
        self.q = (torch.randn(self.rows, Hq, hd, generator=g) * q_scale).to(self.dt)
        self.K, self.V = normal(self.n_pages, Hkv, page, hd), normal(self.n_pages, Hkv, page, hd)
        self.scale = 1 / math.sqrt(hd)

    def raw(self, rows, at):
        import torch
        bits = rows.view(torch.int16).numpy()
        return torch.from_numpy(rows_to_pages(bits, at)).view(self.dt).cuda()

    def call(self, scale=0.0, stream=None, max_fresh=None, q_pad=0, out_pad=0, workspace=None, poison=7.0):
        """-> out [rows, Hq, hd] (float64 on the host); rows nobody has hold `poison`."""
        import torch
        hd, Hq = self.hd, self.Hq
        q = torch.full((self.rows, Hq * hd + q_pad), float("nan"), dtype=self.dt)
        q[:, :Hq * hd] = self.q.view(self.rows, -1)
        self.dev = dict(k=self.raw(self.K, key_at), v=self.raw(self.V, value_at), q=q.cuda(),
                        out=torch.full((self.rows, Hq * hd + out_pad), poison, dtype=self.dt).cuda(),
                        table=torch.from_numpy(self.table).cuda(), row_start=torch.from_numpy(self.row_start).cuda(),
                        seq_len=torch.tensor(self.lens, dtype=torch.int32).cuda())
        d = self.dev
        cache = pkg.StairsPagedCache(k=d["k"].data_ptr(), v=d["v"].data_ptr(), dtype=CODE[self.dtype], n_pages=self.n_pages,
                                     page_size=self.page, n_kv_heads=self.Hkv, head_dim=hd)
        a = pkg.StairsPagedAttention(n_seqs=len(self.lens), max_blocks=self.max_blocks, rows=self.rows, n_heads=Hq,
                                     max_fresh=max(self.fresh) if max_fresh is None else max_fresh, q=d["q"].data_ptr(),
                                     out=d["out"].data_ptr(), q_stride=d["q"].stride(0), out_stride=d["out"].stride(0),
                                     block_table=d["table"].data_ptr(), row_start=d["row_start"].data_ptr(),
                                     seq_len=d["seq_len"].data_ptr(), scale=scale)
        n = pkg.stairs_paged_attention_workspace(cache, a)
        d["work"] = torch.zeros(max(n, 16), dtype=torch.uint8).cuda() if workspace is None else workspace
        a.workspace, a.workspace_bytes = d["work"].data_ptr(), d["work"].numel()
        self.cache, self.args = cache, a
        torch.cuda.synchronize()
        pkg.stairs_paged_attention(cache, a, torch.cuda.current_stream().cuda_stream if stream is None else stream)
        torch.cuda.synchronize()
        return self.result(out_pad, poison)

    def result(self, out_pad=0, poison=7.0):
        out = self.dev["out"].double().cpu()
        if out_pad:
            assert bool((out[:, self.Hq * self.hd:] == poison).all())
        return out[:, :self.Hq * self.hd].reshape(self.rows, self.Hq, self.hd).numpy()

    def reference(self, scale=None):
        return attention_reference(self.q.double().numpy(), self.K.double().numpy(), self.V.double().numpy(), self.table,
                                   self.row_start, self.lens, self.scale if scale is None else scale, HALF_STEP[self.dtype])

    def check(self, out, scale=None, poison=7.0):
        want, tol = self.reference(scale)
        mine = ~np.isnan(want) | (np.arange(self.rows) < self.row_start[-1])[:, None, None]
        assert (out[~mine] == poison).all(), "rows behind the last sequence were written"
        bad = mine & ~(np.isnan(want) & np.isnan(out)) & ~(np.abs(out - want) <= tol) & ~(out == want)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.nanmax(np.where(bad, np.abs(out - want) / tol, 0))))


# ---- sampling ------------------------------------------------------------------------------------------------------
def keep_reference(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(kept mask, weights) of one row of float64 logits."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    if not (x > -np.inf).any():
        return np.zeros(len(x), bool), np.zeros(len(x))
    top = x.max()
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(x == top, 1.0, np.exp((x - top) / float(temperature)))
    w[np.isnan(w)] = 0
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if 0 < top_k < len(x):
        order = order[:top_k]
    if top_p < 1:
        to = np.cumsum(w[order])
        before = np.concatenate([[0.0], to[:-1]])
        stay = before < float(np.float32(top_p)) * to[-1]
        stay[0] = True
        order = order[stay]
    if min_p > 0:
        order = order[w[order] >= min(float(np.float32(min_p)), 1.0)]
    keep = np.zeros(len(x), bool)
    keep[order] = True
    return keep & (w > 0), w


def sample_reference(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, kept)"""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    if not (x > -np.inf).any():
        return -1, -np.inf, 0
    if not temperature > 0:
        return int(np.argmax(x)), 0.0, 1
    keep, w = keep_reference(x, temperature, top_k, top_p, min_p)
    to = np.cumsum(np.where(keep, w, 0.0))
    token = int(np.searchsorted(to, float(np.float32(u)) * to[-1], side="right"))
    if token >= len(x):
        token = int(np.flatnonzero(np.where(keep, w, 0.0))[-1])
    return token, float(np.log(w[token] / to[-1])), int(keep.sum())


def sample_call(logits, dtype, u=None, temperature=None, top_k=None, top_p=None, min_p=None, ld=None, want=("logprob", "kept"), stream=None):
    """logits [rows, vocab] (float32 torch tensor on the host) -> (token, logprob, kept) as numpy arrays"""
    import torch
    n, V = logits.shape
    ld = ld or V
    buf = torch.full((n, ld), float("inf")).to(torch_type(dtype))
    buf[:, :V] = logits.to(torch_type(dtype))
    dev = lambda v, t: None if v is None else torch.as_tensor(np.broadcast_to(np.asarray(v, t), (n,)).copy()).cuda()  # noqa: E731
    d = dict(x=buf.cuda(), t=dev(temperature, np.float32), k=dev(top_k, np.int32), p=dev(top_p, np.float32), m=dev(min_p, np.float32),
             u=dev(u, np.float32), token=torch.full((n,), -7, dtype=torch.int32).cuda(),
             logprob=torch.full((n,), 7.0).cuda() if "logprob" in want else None,
             kept=torch.full((n,), -7, dtype=torch.int32).cuda() if "kept" in want else None)
    at = lambda k: None if d[k] is None else d[k].data_ptr()  # noqa: E731
    a = pkg.StairsSampling(dtype=CODE[dtype], rows=n, vocab=V, ld=ld, logits=at("x"), temperature=at("t"), top_k=at("k"), top_p=at("p"),
                           min_p=at("m"), uniform=at("u"), token=at("token"), logprob=at("logprob"), kept=at("kept"))
    work = torch.zeros(max(16, pkg.stairs_sample_workspace(a)), dtype=torch.uint8).cuda()
    a.workspace, a.workspace_bytes = work.data_ptr(), work.numel()
    torch.cuda.synchronize()
    pkg.stairs_sample_device(a, torch.cuda.current_stream().cuda_stream if stream is None else stream)
    torch.cuda.synchronize()
    host = lambda k: None if d[k] is None else d[k].cpu().numpy()  # noqa: E731
    return host("token"), host("logprob"), host("kept"), buf[:, :V].double().numpy()
