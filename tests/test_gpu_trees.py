"""GPU: trees of drafted tokens: plan, attention, walk, and the caches brought in line; against plain implementations in 64 bits
(trees_util.py)."""
import numpy as np
import pytest

import paper_2407_19947_amd as pkg
import operators_util as ou
import trees_util as tu

pytestmark = pytest.mark.gpu


def i32(v):
    import torch
    return torch.as_tensor(np.asarray(v, np.int32).reshape(-1).copy()).cuda()


def forest(rng, counts):
    """Trees of so many rows; now and then a parent that is none."""
    parent = []
    for n in counts:
        t = tu.random_tree(rng, n) if n else []
        for i in range(1, n):
            if rng.random() < 0.05:
                t[i] = int(rng.choice([-1, -2 ** 31, i, i + 1, 64, 2 ** 31 - 1]))
        parent += t
    return parent


class Trees:
    def __init__(self, counts, lens, spare=5, seed=0, parent=None):
        rng = np.random.default_rng([seed, len(counts), sum(counts)])
        self.counts, self.lens = counts, list(lens)
        self.row_start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.rows = int(self.row_start[-1]) + spare
        self.parent = (forest(rng, counts) if parent is None else list(parent)) + [0] * spare
        self.token = rng.integers(0, 5, self.rows)               # (few different tokens: siblings share some)
        self.predicted = rng.integers(0, 5, self.rows)
        self.token[rng.random(self.rows) < 0.05] = -1

    def plan(self, position=True, stream=None):
        import torch
        B = len(self.counts)
        d = dict(row_start=i32(self.row_start), seq_len=i32(self.lens), parent=i32(self.parent), position=i32([-9] * (self.rows + 3)),
                 sees=torch.full((self.rows + 3,), -9, dtype=torch.int64).cuda())
        t = pkg.StairsTree(n_seqs=B, rows=self.rows, **{k: v.data_ptr() for k, v in d.items()})
        if not position:
            t.position = None
        torch.cuda.synchronize()
        pkg.stairs_tree_plan(t, torch.cuda.current_stream().cuda_stream if stream is None else stream)
        torch.cuda.synchronize()
        return d["position"].cpu().numpy(), d["sees"].cpu().numpy()

    def check_plan(self):
        position, sees = self.plan()
        want_position, want_sees = tu.tree_reference(self.row_start, self.lens, self.parent, self.rows)
        assert position[:self.rows].tolist() == want_position.tolist() and sees[:self.rows].view(np.uint64).tolist() == want_sees.tolist()
        assert (position[self.rows:] == -9).all() and (sees[self.rows:] == -9).all()
        position, again = self.plan(position=False)
        assert (position == -9).all() and np.array_equal(again, sees)

    def walk(self):
        import torch
        B = len(self.counts)
        d = dict(row_start=i32(self.row_start), seq_len=i32(self.lens), parent=i32(self.parent), token=i32(self.token), predicted=i32(self.predicted),
                 kept=i32([-9] * (B + 1)), cached=i32(range(100, 101 + B)), path=i32([-9] * (self.rows + 3)), emitted=i32([-9] * (self.rows + 3)))
        t = pkg.StairsTreeWalk(n_seqs=B, rows=self.rows, **{k: v.data_ptr() for k, v in d.items()})
        torch.cuda.synchronize()
        pkg.stairs_tree_walk(t, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return {k: v.cpu().numpy() for k, v in d.items()}

    def check_walk(self):
        got = self.walk()
        B = len(self.counts)
        kept, cached, path, emitted = tu.walk_reference(self.row_start, self.lens, self.parent, self.token, self.predicted, self.rows, range(100, 100 + B))
        assert got["kept"].tolist() == kept + [-9] and got["cached"].tolist() == cached + [100 + B]
        assert got["path"].tolist() == path.tolist() + [-9] * 3 and got["emitted"].tolist() == emitted.tolist() + [-9] * 3
        return kept


@pytest.mark.parametrize("counts,lens", [
    ([1], [1]), ([7], [300]), ([64], [64]), ([63, 64, 65, 1, 0, 2], [70, 64, 65, 900, 12, 2]), ([5, 200, 64, 0, 33], [5, 1000, 100, 0, 40]),
    ([5, 9, 3, 70], [0, 8, -4, 69]),                             # no pages; fewer positions than rows
])
def test_plan_and_walk_of_chosen_requests(counts, lens):
    for seed in range(4):
        t = Trees(counts, lens, seed=seed)
        t.check_plan()
        t.check_walk()


@pytest.mark.parametrize("B", [1, 3, 4, 5, 257, 1024])
def test_plan_and_walk_of_random_requests(B):
    rng = np.random.default_rng(B)
    counts = np.where(rng.random(B) < 0.1, rng.integers(65, 150, B), rng.integers(0, 65, B))
    lens = counts + rng.integers(0, 3000, B)
    lens[rng.random(B) < 0.1] = 0
    t = Trees(counts.tolist(), lens.tolist(), spare=3000 if B < 10 else 1, seed=B)
    t.check_plan()
    t.check_walk()


def test_walks_to_the_end_of_chains():
    """A chain in which everything fits, one that stops at its first token, the longest chain, prompts' rows that go with their parents."""
    t = Trees([64, 5, 5, 64], [64, 90, 90, 4000], parent=[*range(-1, 63), *range(-1, 4), *range(-1, 4), *range(-1, 63)])
    t.token[:], t.predicted[:] = 3, 3
    t.token[65] = 4
    t.token[74:74 + 64] = -1
    t.predicted[74:] = np.arange(len(t.predicted) - 74)
    t.check_plan()
    assert t.check_walk() == [64, 1, 5, 64]


def test_nothing_but_spare_rows():
    t = Trees([], [], spare=7)
    t.check_plan()
    t.check_walk()
    t = Trees([0, 0], [5, 0], spare=0)
    assert t.check_walk() == [0, 0]


def test_row_starts_that_make_no_sense_stay_in_their_buffers():
    for start in ([0, 2 ** 31 - 1, 5, 3], [-5, 4, 9, 9], [0, 400, 401, 402], [3, 2, 1, 0]):
        t = Trees([3, 3, 3], [10, 10, 10], spare=2)
        t.row_start = np.array(start, np.int32)
        position, sees = t.plan()
        assert (position[t.rows:] == -9).all() and (sees[t.rows:] == -9).all()
        got = t.walk()
        assert (got["path"][t.rows:] == -9).all() and got["kept"][3] == -9 and got["cached"][3] == 103


# ---- attention -----------------------------------------------------------------------------------------------------------
def tree_masks(rng, fresh):
    """What the rows of random trees see; chunks: anything."""
    sees = []
    for n in fresh:
        parent = tu.random_tree(rng, n) if n else []
        sees += [sum(1 << j for j in tu.path_of(parent, i)) if n <= 64 else int(rng.integers(0, 2 ** 63)) for i in range(n)]
    return sees


HEADS = [(4, 4, 64), (4, 4, 128), (8, 2, 64), (8, 2, 128), (7, 1, 128), (40, 2, 64)]


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq,Hkv,hd", HEADS)
@pytest.mark.parametrize("n", [1, 2, 7, 15, 33, 64])
def test_attention_of_trees(n, Hq, Hkv, hd, dtype, held):
    rng = np.random.default_rng([n, Hq, hd])
    lens = [n, n + 1, n + 31, n + 32, 96 + n // 2 + n % 2, 300]
    lens = [max(n, x) for x in lens]
    a = tu.Attend(dtype, lens, [n] * len(lens), Hq, Hkv, hd, [32, 64, 256][n % 3], held=held, sees=tree_masks(rng, [n] * len(lens)), seed=n)
    a.check(a.call())


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_of_trees_of_all_sizes_at_every_border(dtype, held):
    rng = np.random.default_rng(11)
    fresh = [1, 2, 5, 9, 16, 17, 31, 32, 33, 63, 64, 3, 64, 7, 0, 20]
    lens = [f + int(c) for f, c in zip(fresh, [0, 31, 32, 63, 64, 65, 127, 128, 129, 1, 62, 255, 33, 4000, 5, 12])]
    for Hq, Hkv, hd, page in ((4, 4, 64, 32), (8, 2, 128, 64)):
        a = tu.Attend(dtype, lens, fresh, Hq, Hkv, hd, page, held=held, sees=tree_masks(rng, fresh))
        a.check(a.call())


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("Hq,Hkv,hd", [(4, 4, 64), (8, 2, 128)])
def test_attention_of_trees_beside_chunks_and_single_rows(Hq, Hkv, hd, held):
    """Sequences with more than 64 rows are no trees, whatever sees holds for them."""
    rng = np.random.default_rng(2)
    fresh = [1, 64, 65, 200, 12, 1, 128, 30]
    lens = [9000, 100, 65, 700, 500, 1, 300, 30]
    a = tu.Attend("bf16", lens, fresh, Hq, Hkv, hd, 64, held=held, sees=tree_masks(rng, fresh))
    a.check(a.call())


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("n", [5, 40])
def test_a_chain_is_what_causal_rows_see(n, held):
    """Within what both may be off by (the sums' order is the launch's); bits behind a sequence's rows say nothing."""
    lens = [n, 100, 333]
    chain = [(2 << i) - 1 for _ in lens for i in range(n)]
    for dtype, heads in (("bf16", (8, 2, 128)), ("fp16", (2, 2, 64))):
        a = tu.Attend(dtype, lens, [n] * 3, *heads, 64, held=held, seed=n)
        a.check(a.call())
        want, tol = a.reference()
        a.sees = chain
        out = a.call()
        live = a.row_start[-1]
        ou.check_close(out[:live], want[:live], tol[:live])
        a.sees = [s | ~((1 << n) - 1) & (2 ** 64 - 1) for s in chain]
        assert np.array_equal(a.call(), out)


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("n", [4, 64])
def test_masks_of_every_kind(n, held):
    """Rows that see none of the new rows (and nothing at all where there is no context), not themselves, all of them, any of them."""
    rng = np.random.default_rng(n)
    for dtype, heads in (("bf16", (8, 2, 64)), ("fp16", (4, 4, 128))):
        lens = [n, n + 45, n + 200]
        sees = [int(x) for x in rng.integers(0, 2 ** 63, 3 * n)]
        for b in range(3):
            sees[b * n], sees[b * n + 1], sees[b * n + 2], sees[b * n + 3] = 0, 2 ** 64 - 1, 1 << (n - 1), 0
        a = tu.Attend(dtype, lens, [n] * 3, *heads, 32, held=held, sees=sees, seed=n)
        out = a.call()
        a.check(out)
        assert (out[0] == 0).all() and (out[3] == 0).all() and (out[n] != 0).any()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,Hq,Hkv,hd", [(6, 8, 2, 128), (6, 4, 4, 64), (50, 8, 2, 128)])
def test_rows_of_other_branches_may_hold_anything(n, Hq, Hkv, hd, value):
    """A row's keys and values that are no numbers show in the rows that see it alone."""
    import torch
    parent = [-1] + [0, 0, 1, 2, 2] + list(range(5, n - 1))
    sees = [sum(1 << j for j in tu.path_of(parent, i)) for i in range(n)] * 2
    for dtype in ("bf16", "fp16"):
        a = tu.Attend(dtype, [n + 70, n + 3], [n, n], Hq, Hkv, hd, 32, held=False, sees=sees)
        clean = a.call()
        a.check(clean)
        for T in (a.K, a.V):
            for b, m in enumerate(a.lens):
                at = m - n + 1                                   # row 1 and, behind it, row 3
                T[a.table[b, at // 32], :, at % 32] = value
        out = a.call()
        off = np.array([sees[i] >> 1 & 1 for i in range(n)] * 2, bool)
        assert off.sum() == 4 and np.array_equal(out[:2 * n][~off], clean[:2 * n][~off]) and not np.isfinite(out[:2 * n][off]).any()


def test_trees_with_more_rows_than_positions_and_positions_than_blocks():
    a = tu.Attend("fp16", [3, 40, 200], [7, 60, 2], 8, 2, 64, 32, held=False, extra_blocks=0, sees=tree_masks(np.random.default_rng(1), [7, 60, 2]))
    a.check(a.call())                                            # rows in front of position 0 are nowhere
    a = tu.Attend("bf16", [64, 96], [2, 40], 8, 2, 64, 32, held=True, extra_blocks=0, sees=[3, 3] * 21)
    a.lens = [10 ** 9, 10 ** 9 + 5]                              # behind the table's three blocks nothing is seen
    out = a.call()
    K, V = a.numbers()
    want, tol = tu.attention_reference(a.q.double().numpy(), K, V, a.table, a.row_start, [98, 136], a.scale, ou.HALF_STEP["bf16"], tu.TWO["bf16"], ou.HALF_STEP["bf16"])
    live = a.row_start[-1]
    ou.check_close(out[:live], want[:live], tol[:live])


def test_trees_with_strides_hints_and_a_scale():
    rng = np.random.default_rng(4)
    fresh = [30, 3, 5, 64]
    a = tu.Attend("bf16", [300, 64, 5, 900], fresh, 8, 2, 128, 64, held=True, sees=tree_masks(rng, fresh))
    a.check(a.call(scale=0.3, q_pad=40, out_pad=8), scale=0.3)
    for hint in (0, 1, 10, 5000):
        a.check(a.call(max_fresh=hint))


def test_calls_with_and_without_trees_share_a_workspace():
    import torch
    rng = np.random.default_rng(8)
    calls = [tu.Attend("bf16", [9000, 3000, 64], [12, 64, 2], 8, 2, 128, 64, held=h, sees=s) for h in (False, True) for s in (None, tree_masks(rng, [12, 64, 2]))]
    alone = [x.call() for x in calls]
    for x, y in zip(calls, alone):
        x.check(y)
    work = torch.zeros(max(x.dev["work"].numel() for x in calls), dtype=torch.uint8).cuda()
    for i in (0, 1, 2, 3, 3, 1, 0, 2):
        assert np.array_equal(calls[i].call(workspace=work), alone[i]), i


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("lens,n", [([3000], 40), ([12000], 64), ([2500, 700, 9000], 33), ([1100] * 4, 64), ([6000, 64, 64, 64, 64], 64)])
def test_attention_of_trees_whose_tiles_are_cut_into_any_number_of_pieces(lens, n, held):
    """Pieces are joined two at a time: 2 and more of them, powers of two and others; twice on one workspace with the same bits, every
    ticket 0 again."""
    import torch
    rng = np.random.default_rng(n)
    for dtype, heads in (("bf16", (4, 1, 128)), ("fp16", (6, 2, 64))):
        a = tu.Attend(dtype, lens, [n] * len(lens), *heads, 64, held=held, sees=tree_masks(rng, [n] * len(lens)), seed=n)
        out = a.call()
        a.check(out)
        work = torch.zeros_like(a.dev["work"])
        for _ in range(3):
            assert np.array_equal(a.call(workspace=work), out)
        assert int(work[:8192].sum()) == 0


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("B", [2, 63, 64, 65, 130, 1000])
def test_attention_of_trees_of_many_sequences(B, held):
    """Long ones among short ones, before and behind the first 64; sequences without rows."""
    rng = np.random.default_rng([B, held])
    fresh = rng.integers(0, 4, B)
    lens = fresh + rng.integers(0, 60, B)
    for at, n, f in ((0, 3000, 64), (B // 2, 900, 40), (B - 1, 5000, 20), (B * 3 // 4, 2000, 3)):
        lens[at], fresh[at] = n, f
    a = tu.Attend("bf16", lens.tolist(), fresh.tolist(), 4, 2, 64, 32, held=held, sees=tree_masks(rng, fresh.tolist()), seed=B)
    a.check(a.call())


def test_two_calls_at_once_with_a_workspace_each():
    import torch
    rng = np.random.default_rng(6)
    a = tu.Attend("bf16", [9000, 3000], [64, 33], 8, 2, 128, 64, held=False, sees=tree_masks(rng, [64, 33]))
    b = tu.Attend("fp16", [2000, 6000], [60, 64], 8, 2, 128, 64, held=True, sees=tree_masks(rng, [60, 64]))
    first = [a.call(), b.call()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for x in (a, b):
        x.dev["out"].fill_(7.0)
    torch.cuda.synchronize()
    for _ in range(5):
        for x, st in zip((a, b), streams):
            pkg.stairs_paged_attention(x.cache, x.args, st.cuda_stream)
    torch.cuda.synchronize()
    for x, want in zip((a, b), first):
        assert np.array_equal(x.result(), want)


def test_plans_walks_and_moves_on_a_stream_of_the_callers():
    import torch
    side = torch.cuda.Stream()
    t = Trees([7, 64, 1], [70, 64, 5])
    one, two = t.plan(), t.plan(stream=side.cuda_stream)
    assert all(np.array_equal(x, y) for x, y in zip(one, two))
    L = Layers("bf16", 2, 4, 32, 2, 64, False)
    L.check(np.array([[2, 0, 3, 1]], np.int32), [0, 40], [100], paths(np.random.default_rng(3), [40])[0], [12], stream=side.cuda_stream)


# ---- the caches in line with a path ----------------------------------------------------------------------------------------
class Layers:
    def __init__(self, dtype, layers, n_pages, page, Hkv, hd, held, seed=0):
        import torch
        rng = np.random.default_rng([seed, layers, n_pages])
        self.held, self.page, self.Hkv, self.hd, self.n_pages = held, page, Hkv, hd, n_pages
        n, e = page * hd, 1 if held else 2
        u8 = lambda *s: rng.integers(0, 256, s).astype(np.uint8)  # noqa: E731   (any bits: they are moved, not computed with)
        self.k, self.v, self.s = u8(layers, n_pages, Hkv, n * e), u8(layers, n_pages, Hkv, n * e), u8(layers, n_pages, Hkv, page * 2)
        self.dev = [torch.from_numpy(a.copy()).cuda() for a in (self.k, self.v, self.s)]
        self.caches = [pkg.StairsPagedCache(k=self.dev[0][i].data_ptr(), v=self.dev[1][i].data_ptr(), dtype=ou.CODE[dtype], n_pages=n_pages, page_size=page,
                                            n_kv_heads=Hkv, head_dim=hd, held=pkg.DTYPE_E4M3 if held else 0, scale=self.dev[2][i].data_ptr() if held else None)
                       for i in range(layers)]

    def places(self):
        p, e = np.meshgrid(np.arange(self.page), np.arange(self.hd), indexing="ij")
        p0 = np.arange(self.page)
        if self.held:
            return tu.held_key_at(p, e, self.hd), tu.held_value_at(p, e, self.hd), np.stack([tu.held_scale_at(p0, 0), tu.held_scale_at(p0, 1)], 1)
        return ou.key_at(p, e, self.hd), ou.value_at(p, e, self.hd), None

    def moved(self, table, row_start, seq_len, path, kept):
        """The pools as they are to be: every row read from what was there before the call."""
        out = [a.copy() for a in (self.k, self.v, self.s)]
        places = self.places()
        for b in range(len(seq_len)):
            n, r0 = row_start[b + 1] - row_start[b], row_start[b]
            if n > 64 or n == 0 or seq_len[b] < n:
                continue
            for j in range(min(kept[b], n)):
                frm, to = seq_len[b] - n + path[r0 + j], seq_len[b] - n + j
                if frm == to or not 0 <= path[r0 + j] < n:
                    continue
                blocks = [table[b, x // self.page] if x // self.page < table.shape[1] else -1 for x in (frm, to)]
                if not all(0 <= x < self.n_pages for x in blocks):
                    continue
                for i, (src, dst) in enumerate(zip((self.k, self.v, self.s), out)):
                    if places[i] is None:
                        continue
                    w = 1 if self.held else 2
                    x, y = src.reshape(*src.shape[:3], -1, w), dst.reshape(*dst.shape[:3], -1, w)
                    y[:, blocks[1], :, places[i][to % self.page]] = x[:, blocks[0], :, places[i][frm % self.page]]
        return out

    def check(self, table, row_start, seq_len, path, kept, stream=None):
        import torch
        p = dict(block_table=i32(table), row_start=i32(row_start), seq_len=i32(seq_len), path=i32(path), kept=i32(kept))
        a = pkg.StairsPagedPath(n_seqs=len(seq_len), max_blocks=table.shape[1], rows=len(path), **{k: v.data_ptr() for k, v in p.items()})
        torch.cuda.synchronize()
        pkg.stairs_paged_compact(self.caches, a, torch.cuda.current_stream().cuda_stream if stream is None else stream)
        torch.cuda.synchronize()
        for got, want in zip(self.dev, self.moved(table, row_start, seq_len, path, kept)):
            got = got.cpu().numpy()
            assert np.array_equal(got, want), np.argwhere(got != want)[:4]


def paths(rng, counts):
    path, kept = [], []
    for n in counts:
        if n == 0 or n > 64:
            path += list(range(n))
            kept.append(n)
            continue
        k = int(rng.integers(1, min(n, 12) + 1)) if rng.random() < 0.9 else n
        p = [0] + sorted(rng.choice(np.arange(1, n), k - 1, replace=False).tolist()) if n > 1 else [0]
        path += p + [-1] * (n - len(p))
        kept.append(len(p))
    return path, kept


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("Hkv,hd,page,layers", [(4, 64, 32, 3), (2, 128, 64, 1), (7, 128, 32, 2), (1, 64, 256, 5)])
def test_compact(Hkv, hd, page, layers, held):
    rng = np.random.default_rng([Hkv, hd, page])
    for it in range(3):
        counts = rng.permutation([1, 2, 3, 15, 30, 64, 64, 0, 65, 7]).tolist()
        lens = [n + int(rng.integers(0, 200)) for n in counts]
        held_pages = [-(-n // page) for n in lens]
        L = Layers("bf16", layers, sum(held_pages) + 1, page, Hkv, hd, held, seed=it)
        order = rng.permutation(L.n_pages)
        table = np.full((len(counts), max(held_pages) + 1), -1, np.int32)
        at = 0
        for b, n in enumerate(held_pages):
            table[b, :n] = order[at:at + n]
            at += n
        row_start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        path, kept = paths(rng, counts)
        if it == 2:                                              # nothing of the first requests: no pages, a page that is none
            lens[0], table[1, -2:] = 0, L.n_pages
            table[2, 0] = -7
        L.check(table, row_start, lens, path + [-1] * 3, kept)


def test_compact_of_more_pools_than_a_launch_has_addresses_for():
    rng = np.random.default_rng(0)
    L = Layers("fp16", 131, 4, 32, 2, 64, False)
    L.check(np.array([[2, 0, 3, 1]], np.int32), [0, 40], [100], paths(rng, [40])[0], [12])


@pytest.mark.parametrize("held", [False, True])
def test_compact_beyond_32_bit_offsets(held):
    """The last pages of pools of more than 2^32 bytes each; rows stored there, moved, and read back."""
    import torch
    page, hd, n_pages = 256, 128, 140000 if held else 70000
    bytes_ = [page * hd * (1 if held else 2)] * 2 + [page * 2]
    pools = [torch.zeros(n_pages, n, dtype=torch.uint8, device="cuda") for n in bytes_]
    cache = pkg.StairsPagedCache(k=pools[0].data_ptr(), v=pools[1].data_ptr(), dtype=pkg.DTYPE_BF16, n_pages=n_pages, page_size=page, n_kv_heads=1, head_dim=hd,
                                 held=pkg.DTYPE_E4M3 if held else 0, scale=pools[2].data_ptr())
    n, context = 20, 250                                         # across a page's end
    table = np.array([[n_pages - 1, n_pages - 2]], np.int32)
    pos = context + np.arange(n)
    slot = i32(table[0, pos // page] * page + pos % page)
    x = torch.randn(2, n, hd, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    pkg.stairs_paged_append(cache, pkg.StairsPagedRows(rows=n, n_heads=0, k=x[0].data_ptr(), v=x[1].data_ptr(), k_stride=hd, v_stride=hd, slot=slot.data_ptr(), rope_theta=0.0), None)
    got = [torch.zeros(2, n, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    reads = [pkg.StairsPagedRead(rows=n, k=g[0].data_ptr(), v=g[1].data_ptr(), k_stride=hd, v_stride=hd, slot=slot.data_ptr()) for g in got]
    pkg.stairs_paged_read(cache, reads[0], None)
    path = [0, 3, 7, 8, 13, 14, 15, 19]
    p = dict(block_table=i32(table), row_start=i32([0, n]), seq_len=i32([context + n]), path=i32(path + [-1] * (n - len(path))), kept=i32([len(path)]))
    pkg.stairs_paged_compact([cache], pkg.StairsPagedPath(n_seqs=1, max_blocks=2, rows=n, **{k: v.data_ptr() for k, v in p.items()}), None)
    pkg.stairs_paged_read(cache, reads[1], None)
    torch.cuda.synchronize()
    want = got[0].clone()
    want[:, :len(path)] = got[0][:, path]
    assert torch.equal(got[1], want) and bool((got[0] != 0).any(2).all())


def test_compact_with_paths_that_make_no_sense_stays_in_its_pages():
    L = Layers("bf16", 1, 3, 32, 2, 64, True)
    table = np.array([[2, 0]], np.int32)
    for path, kept, lens in (([0, 70, -3, 2 ** 31 - 1, 4, 5], [6], [40]), ([0] * 6, [2 ** 31 - 1], [64]), ([0, 2, 4, 5, -1, -1], [-4], [64]),
                             ([0, 2, 3, 4, 5, -1], [5], [2 ** 31 - 1]), ([0, 2, 3, 4, 5, -1], [5], [66])):
        import torch
        p = dict(block_table=i32(table), row_start=i32([0, 6]), seq_len=i32(lens), path=i32(path), kept=i32(kept))
        a = pkg.StairsPagedPath(n_seqs=1, max_blocks=2, rows=6, **{k: v.data_ptr() for k, v in p.items()})
        pkg.stairs_paged_compact(L.caches, a, None)
        torch.cuda.synchronize()
        assert np.array_equal(L.dev[0][0, 1].cpu().numpy(), L.k[0, 1])     # the page nobody has


# ---- as they are used ------------------------------------------------------------------------------------------------------
class Server:
    """Requests over one pool a layer; a step is plan, tree plan, store, attend, draw, walk, compact, on the program's buffers.

    The model: a token has queries, keys and values of its own in each layer; the logits are the layers' attention outputs, summed, times a table of
    token vectors."""

    def __init__(self, dtype, held, B, layers=2, Hq=8, Hkv=2, hd=64, page=32, n_pages=60, most=20, cap=160, vocab=24, longest=170, seed=0):
        import torch
        self.dtype, self.B, self.layers, self.Hq, self.Hkv, self.hd, self.cap, self.vocab, self.page = dtype, B, layers, Hq, Hkv, hd, cap, vocab, page
        self.dt = dt = ou.torch_type(dtype)
        g = torch.Generator().manual_seed(seed)
        wide = (Hq + 2 * Hkv) * hd
        self.rows_of = torch.randn(layers, vocab, wide, generator=g).to(dt).cuda()
        self.vectors = torch.randn(vocab, Hq * hd, generator=g).cuda()
        z = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")  # noqa: E731
        self.t = t = dict(cached=z(B), fresh=z(B), held=z(B), n_free=z(1), table=z(B, most), free=torch.arange(n_pages, dtype=torch.int32).cuda(), row_start=z(B + 1), seq_len=z(B),
                          at=z(cap), slot=z(cap), parent=z(cap), ids=z(cap), token=z(cap), position=z(cap), sees=torch.zeros(cap, dtype=torch.int64, device="cuda"),
                          predicted=z(cap), kept=z(B), path=z(cap), emitted=z(cap))
        t["n_free"].fill_(n_pages)
        ptr = {k: v.data_ptr() for k, v in t.items()}
        self.caches = self.new_caches(held, n_pages)
        self.plan = pkg.StairsPagePlan(n_seqs=B, max_blocks=most, n_pages=n_pages, page_size=page, max_rows=cap, cached=ptr["cached"], fresh=ptr["fresh"],
                                       held=ptr["held"], n_free=ptr["n_free"], block_table=ptr["table"], free_pages=ptr["free"], held_out=ptr["held"],
                                       n_free_out=ptr["n_free"], row_start=ptr["row_start"], seq_len=ptr["seq_len"], position=ptr["at"], slot=ptr["slot"])
        self.tree = pkg.StairsTree(n_seqs=B, rows=cap, row_start=ptr["row_start"], seq_len=ptr["seq_len"], parent=ptr["parent"], position=ptr["position"], sees=ptr["sees"])
        self.walk = pkg.StairsTreeWalk(n_seqs=B, rows=cap, row_start=ptr["row_start"], seq_len=ptr["seq_len"], parent=ptr["parent"], token=ptr["token"],
                                       predicted=ptr["predicted"], kept=ptr["kept"], cached=ptr["cached"], path=ptr["path"], emitted=ptr["emitted"])
        self.path = pkg.StairsPagedPath(n_seqs=B, max_blocks=most, rows=cap, block_table=ptr["table"], row_start=ptr["row_start"], seq_len=ptr["seq_len"], path=ptr["path"],
                                        kept=ptr["kept"])
        self.qkv = torch.zeros(layers, cap, wide, dtype=dt, device="cuda")
        self.q, self.out = (torch.zeros(layers, cap, Hq * hd, dtype=dt, device="cuda") for _ in range(2))
        self.logits, self.cold = torch.zeros(cap, vocab, device="cuda"), torch.zeros(cap, device="cuda")
        self.rows = [self.rows_arg(self.qkv[i], self.q[i], t["position"], t["slot"]) for i in range(layers)]
        self.attn = [pkg.StairsPagedAttention(n_seqs=B, max_blocks=most, rows=cap, n_heads=Hq, max_fresh=64, q=self.q[i].data_ptr(), out=self.out[i].data_ptr(),
                                              q_stride=Hq * hd, out_stride=Hq * hd, block_table=ptr["table"], row_start=ptr["row_start"], seq_len=ptr["seq_len"],
                                              scale=0.0, sees=ptr["sees"]) for i in range(layers)]
        self.work = torch.zeros(pkg.stairs_paged_attention_workspace(self.caches[0], self.attn[0]), dtype=torch.uint8, device="cuda")
        for a in self.attn:
            a.workspace, a.workspace_bytes = self.work.data_ptr(), self.work.numel()
        self.draw = pkg.StairsSampling(dtype=pkg.DTYPE_FP32, rows=cap, vocab=vocab, ld=vocab, logits=self.logits.data_ptr(), temperature=self.cold.data_ptr(),
                                       token=ptr["predicted"])
        self.swork = torch.zeros(max(16, pkg.stairs_sample_workspace(self.draw)), dtype=torch.uint8, device="cuda")
        self.draw.workspace, self.draw.workspace_bytes = self.swork.data_ptr(), self.swork.numel()
        self.every_row(held, longest)

    def new_caches(self, held, n_pages):
        import torch
        n = self.page * self.hd * (1 if held else 2)
        pools = [torch.zeros(self.layers, n_pages, self.Hkv, m, dtype=torch.uint8, device="cuda") for m in (n, n, self.page * 2)]
        self.keep = getattr(self, "keep", []) + pools
        return [pkg.StairsPagedCache(k=pools[0][i].data_ptr(), v=pools[1][i].data_ptr(), dtype=ou.CODE[self.dtype], n_pages=n_pages, page_size=self.page,
                                     n_kv_heads=self.Hkv, head_dim=self.hd, held=pkg.DTYPE_E4M3 if held else 0, scale=pools[2][i].data_ptr()) for i in range(self.layers)]

    def rows_arg(self, qkv, q_out, position, slot):
        Hq, Hkv, hd, base, e = self.Hq, self.Hkv, self.hd, qkv.data_ptr(), qkv.element_size()
        return pkg.StairsPagedRows(rows=len(qkv), n_heads=Hq, q=base, k=base + Hq * hd * e, v=base + (Hq + Hkv) * hd * e, q_out=q_out.data_ptr(), q_stride=qkv.stride(0),
                                   k_stride=qkv.stride(0), v_stride=qkv.stride(0), q_out_stride=q_out.stride(0), position=position.data_ptr(), slot=slot.data_ptr(),
                                   rope_theta=10000.0)

    def read(self, cache, slots):
        import torch
        k, v = torch.zeros(2, len(slots), self.Hkv * self.hd, dtype=self.dt, device="cuda")
        slot = i32(slots)
        pkg.stairs_paged_read(cache, pkg.StairsPagedRead(rows=len(slots), k=k.data_ptr(), v=v.data_ptr(), k_stride=k.stride(0), v_stride=v.stride(0), slot=slot.data_ptr()), None)
        torch.cuda.synchronize()
        return [x.double().cpu().numpy().reshape(len(slots), self.Hkv, self.hd) for x in (k, v)]

    def every_row(self, held, longest):
        """What each token's row is at each position, by storing and reading them all: q, k, v [layer][position * vocab + token]"""
        import torch
        n = longest * self.vocab
        caches = self.new_caches(held, -(-n // self.page))
        at = np.arange(n)
        self.of = []
        for i, c in enumerate(caches):
            qkv, q = self.rows_of[i].repeat(longest, 1), torch.zeros(n, self.Hq * self.hd, dtype=self.dt, device="cuda")
            position, slot = i32(at // self.vocab), i32(at)
            torch.cuda.synchronize()
            pkg.stairs_paged_append(c, self.rows_arg(qkv, q, position, slot), None)
            torch.cuda.synchronize()
            self.of.append((q.double().cpu().numpy().reshape(n, self.Hq, self.hd), *self.read(c, at)))

    def attended(self, i, seq):
        """Layer i's attention of the last token of seq over all of it, and what the device's may be off by"""
        rows = np.arange(len(seq)) * self.vocab + np.array(seq)
        q, k, v = self.of[i][0][rows[-1:]], self.of[i][1][rows], self.of[i][2][rows]
        half = ou.HALF_STEP[self.dtype]
        want, tol = tu.attention_reference(q, k[None].swapaxes(1, 2), v[None].swapaxes(1, 2), np.zeros((1, 1), int), [0, 1], [len(seq)], 1 / np.sqrt(self.hd), half,
                                           half, half)
        return want[0], tol[0]

    def says(self, seq):
        x = sum(self.attended(i, seq)[0] for i in range(self.layers)).reshape(-1)
        return int(np.argmax(self.vectors.double().cpu().numpy() @ x))

    def step(self, stream):
        pkg.stairs_paged_plan(self.plan, stream)
        pkg.stairs_tree_plan(self.tree, stream)
        ids = self.t["ids"].long()
        for i in range(self.layers):
            self.qkv[i].copy_(self.rows_of[i][ids])
            pkg.stairs_paged_append(self.caches[i], self.rows[i], stream)
            pkg.stairs_paged_attention(self.caches[i], self.attn[i], stream)
        self.logits.copy_((self.out.float().sum(0)[:, None] * self.vectors[None]).sum(2))
        pkg.stairs_sample_device(self.draw, stream)
        pkg.stairs_tree_walk(self.walk, stream)
        pkg.stairs_paged_compact(self.caches, self.path, stream)

    def put(self, trees):
        """For each request (tokens, parents, whether the walk takes them as they are) of its new rows."""
        ids = [x for tok, _, _ in trees for x in tok]
        pad = [0] * (self.cap - len(ids))
        self.t["ids"].copy_(i32(ids + pad))
        self.t["token"].copy_(i32([-1 if forced else x for tok, _, forced in trees for x in tok] + pad))
        self.t["parent"].copy_(i32([x for _, par, _ in trees for x in par] + pad))
        self.t["fresh"].copy_(i32([len(tok) for tok, _, _ in trees]))


def chain(tokens, forced):
    return list(tokens), list(range(-1, len(tokens) - 1)), forced


def drafted(rng, server, seq):
    """The last token of seq and a tree behind it: some branches at random, among them what will be said up to a wrong token."""
    tok, par, tip, n = [seq[-1]], [-1], 0, int(rng.integers(1, 24))
    true, right = list(seq), int(rng.integers(0, 7))
    for _ in range(n):
        if right and rng.random() < 0.6:
            true.append(server.says(true))
            tok.append(true[-1])
            par.append(tip)
            tip, right = len(tok) - 1, right - 1
        else:
            par.append(int(rng.integers(0, len(tok))))
            tok.append(int(rng.integers(0, server.vocab)))
    return tok, par, False


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_steps_of_a_server_that_verifies_trees_captured_and_replayed(dtype, held):
    """Prompts (a chunk, a chain that is forced) and then trees, one graph replay a step.  Every row's attention is that over its own path;
    tokens and paths are what the walk gives for the device's predictions; the caches hold the accepted tokens' rows, bit for bit, as if each had been
    stored alone."""
    import torch
    rng = np.random.default_rng(5)
    B = 3
    server = Server(dtype, held, B)
    server.step(torch.cuda.current_stream().cuda_stream)         # no rows yet: the kernels are loaded
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        server.step(torch.cuda.current_stream().cuda_stream)
    seqs = [rng.integers(0, server.vocab, n).tolist() for n in (5, 70, 33)]
    cached, longest = [0] * B, 0
    for it in range(9):
        trees = [chain(s, True) for s in seqs] if it == 0 else [drafted(rng, server, s) for s in seqs]
        if it == 4:
            trees[1] = ([], [], False)                           # a request that waits
        server.put(trees)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        t = {k: v.cpu().numpy() for k, v in server.t.items()}
        out = server.out.double().cpu().numpy().reshape(server.layers, server.cap, server.Hq, server.hd)
        start = t["row_start"]
        kept, now, path, emitted = tu.walk_reference(start, t["seq_len"], t["parent"], t["token"], t["predicted"], server.cap, cached)
        assert t["kept"].tolist() == kept and t["cached"].tolist() == now
        assert t["path"].tolist() == path.tolist() and t["emitted"].tolist() == emitted.tolist()
        for b, (tok, par, forced) in enumerate(trees):
            front = [] if it == 0 else seqs[b][:-1]
            assert len(front) == cached[b]
            for i in range(len(tok)):
                if it == 0 and i % 7:
                    continue                                     # (every seventh row of the prompts)
                mine = front + [tok[j] for j in (tu.path_of(par, i) if len(tok) <= 64 else range(i + 1))]
                for layer in range(server.layers):
                    want, tol = server.attended(layer, mine)
                    ou.check_close(out[layer, start[b] + i], want, tol, (it, b, i, layer))
            if not tok:
                continue
            got = emitted[start[b]:start[b] + kept[b]].tolist()
            if it == 0:
                assert kept[b] == len(tok)
                seqs[b] = seqs[b] + got[-1:]
            else:
                seqs[b] = seqs[b] + got
                longest = max(longest, kept[b])
            assert now[b] == len(seqs[b]) - 1
        cached = now
        for b in range(B):
            pos = np.arange(cached[b])
            slots = t["table"][b, pos // server.page] * server.page + pos % server.page
            for layer in range(server.layers):
                k, v = server.read(server.caches[layer], slots)
                rows = pos * server.vocab + np.array(seqs[b][:cached[b]])
                assert np.array_equal(k, server.of[layer][1][rows]) and np.array_equal(v, server.of[layer][2][rows]), (it, b, layer)
    assert longest > 3                                           # some paths were long


# ---- what a call leaves alone ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_compact_writes_the_aligned_fours_that_rows_move_to_and_nothing_else(hd, held):
    """Four requests with a page, each at eight positions of its own, and rows stored by another stream at the last of them: whoever wrote more than
    the four positions that its rows move to would undo what the others do."""
    import torch
    page, Hkv, layers, n_pages = 32, 6, 20, 40
    L = Layers("bf16", layers, n_pages, page, Hkv, hd, held, seed=hd)
    table = np.repeat(np.arange(n_pages, dtype=np.int32)[::-1].copy(), 4)[:, None]
    B = len(table)
    seq_len = [8 * (b % 4) + 7 for b in range(B)]                # seven new rows each, behind 0, 8, 16 and 24 positions
    path, kept = [0, 2, 4, 5, -1, -1, -1] * B, [4, 3, 4, 2] * n_pages
    slots = i32(np.arange(n_pages) * page + 31)
    x = torch.randn(n_pages, 2 * Hkv * hd, generator=torch.Generator().manual_seed(hd)).to(torch.bfloat16).cuda()
    rows = pkg.StairsPagedRows(rows=n_pages, n_heads=0, k=x.data_ptr(), v=x[:, Hkv * hd:].data_ptr(), k_stride=2 * Hkv * hd, v_stride=2 * Hkv * hd, slot=slots.data_ptr(),
                               rope_theta=0.0)
    p = dict(block_table=i32(table), row_start=i32(range(0, 7 * B + 1, 7)), seq_len=i32(seq_len), path=i32(path), kept=i32(kept))
    a = pkg.StairsPagedPath(n_seqs=B, max_blocks=1, rows=7 * B, **{k: v.data_ptr() for k, v in p.items()})
    start = [t.clone() for t in L.dev]
    for c in L.caches:                                           # what the stored rows are alone
        pkg.stairs_paged_append(c, rows, None)
    torch.cuda.synchronize()
    L.k, L.v, L.s = (t.cpu().numpy() for t in L.dev)
    want = L.moved(table, [7 * b for b in range(B + 1)], seq_len, path, kept)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for t, first in zip(L.dev, start):
            t.copy_(first)
        torch.cuda.synchronize()
        pkg.stairs_paged_compact(L.caches, a, streams[0].cuda_stream)
        for c in L.caches:
            pkg.stairs_paged_append(c, rows, streams[1].cuda_stream)
        torch.cuda.synchronize()
        for got, w in zip(L.dev, want):
            got = got.cpu().numpy()
            assert np.array_equal(got, w), np.argwhere(got != w)[:4]


@pytest.mark.parametrize("counts", [[5, 9, 3], [5, 70, 3], [5, 0, 40]])
def test_the_walk_keeps_nothing_of_requests_whose_rows_the_buffers_do_not_hold(counts):
    """A step with more rows than the buffers have: those requests' counts of cached positions stay, so the next step brings their rows again."""
    t = Trees(counts, [300, 200, 100])
    t.rows = 7
    got = t.walk()
    r0 = [0, 5, 5 + counts[1]]
    kept, cached, path, emitted = tu.walk_reference(r0[:2], [300], t.parent, t.token, t.predicted, 7, [100])
    whole = counts[1] == 0                                       # (no rows: all that is cached is its length)
    assert got["kept"].tolist() == kept + [0, 0, -9] and got["cached"].tolist() == cached + [200 if whole else 101, 102, 103]
    assert got["path"].tolist()[:5] == path[:5].tolist() and got["emitted"].tolist()[:5] == emitted[:5].tolist()
    assert (got["path"][7:] == -9).all() and (got["emitted"][7:] == -9).all()


@pytest.mark.parametrize("value", [0x7F, 0xFF])
@pytest.mark.parametrize("n,Hq,Hkv,hd", [(6, 8, 2, 128), (6, 4, 4, 64), (50, 8, 2, 128)])
def test_rows_of_other_branches_may_hold_anything_in_8_bit_pages(n, Hq, Hkv, hd, value):
    """Codes that are no number show in the rows that see them alone, and so do numbers past the type's largest."""
    parent = [-1] + [0, 0, 1, 2, 2] + list(range(5, n - 1))
    sees = [sum(1 << j for j in tu.path_of(parent, i)) for i in range(n)] * 2
    off = np.array([sees[i] >> 1 & 1 for i in range(n)] * 2, bool)
    assert off.sum() == 4
    for dtype, past in (("bf16", 250), ("fp16", 137)):
        a = tu.Attend(dtype, [n + 70, n + 3], [n, n], Hq, Hkv, hd, 32, sees=sees)
        clean = a.call()
        a.check(clean)
        want, tol = a.reference()
        keep = a.kc.copy(), a.vc.copy(), a.vb.copy()
        for kind in ("keys", "values", "past"):
            a.kc, a.vc, a.vb = (x.copy() for x in keep)
            for b, m in enumerate(a.lens):
                at = m - n + 1                                   # row 1 and, behind it, row 3
                page, p = a.table[b, at // 32], at % 32
                if kind == "past":
                    a.vc[page, :, p], a.vb[page, :, p] = 0x7E, past
                else:
                    (a.kc if kind == "keys" else a.vc)[page, :, p] = value
            out = a.call()
            assert not np.isfinite(out[:2 * n][off]).any(), (dtype, kind)
            if kind == "past":                                   # (maxima follow at once there: the same but for the sums' order)
                assert np.isposinf(out[:2 * n][off]).all()
                ou.check_close(out[:2 * n][~off], want[:2 * n][~off], tol[:2 * n][~off], dtype)
            else:
                assert np.array_equal(out[:2 * n][~off], clean[:2 * n][~off]), (dtype, kind)


@pytest.mark.parametrize("held", [False, True])
def test_paths_that_make_no_sense_touch_no_page_of_others(held):
    """Keys, values and powers of two of the page nobody has, and whatever lies in front of the new rows' first aligned four."""
    for path, kept, lens in (([0, 70, -3, 2 ** 31 - 1, 4, 5], [6], [40]), ([0] * 6, [2 ** 31 - 1], [64]), ([0, 2, 4, 5, -1, -1], [-4], [64]),
                             ([0, 2, 3, 4, 5, -1], [5], [2 ** 31 - 1]), ([0, 2, 3, 4, 5, -1], [5], [66]), ([5, 4, 3, 2, 1, 0], [6], [40])):
        L = Layers("bf16", 2, 3, 32, 2, 64, held)
        table = np.array([[2, 0]], np.int32)
        p = dict(block_table=i32(table), row_start=i32([0, 6]), seq_len=i32(lens), path=i32(path), kept=i32(kept))
        a = pkg.StairsPagedPath(n_seqs=1, max_blocks=2, rows=6, **{k: v.data_ptr() for k, v in p.items()})
        import torch
        torch.cuda.synchronize()
        pkg.stairs_paged_compact(L.caches, a, None)
        torch.cuda.synchronize()
        front = (lens[0] - 6) // 4 * 4
        for i, (got, was) in enumerate(zip(L.dev, (L.k, L.v, L.s))):
            got = got.cpu().numpy()
            assert np.array_equal(got[:, 1], was[:, 1]), (path, i)
            places = L.places()[i]
            if places is None:
                assert np.array_equal(got, was)
                continue
            w = 1 if held else 2
            pages = [x.reshape(*x.shape[:3], -1, w)[..., places, :] for x in (got, was)]     # [layer, page, head, position, ...]
            for block, page in enumerate(table[0]):
                mine = np.arange(32) + 32 * block < front
                assert np.array_equal(pages[0][:, page][:, :, mine], pages[1][:, page][:, :, mine]), (path, i, block)
