"""sp_pages_* against a plain model of the table: every array exactly, copied rows bit for bit, nothing else touched."""
import numpy as np
import pytest
import torch

import paper_2507_11830_amd as sp

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def pages_of(n):
    return -(-n // 16) if n > 0 else 0


class Model:
    """The rules, one entry at a time."""

    def __init__(self, rows, width, pages):
        self.table, self.lens, self.refs = np.full((rows, width), -1), np.zeros(rows, int), np.zeros(pages, int)

    def free(self):
        return list(np.flatnonzero(self.refs == 0))

    def reserve(self, rows, new):
        width = self.table.shape[1]
        do = [(r, n) for r, n in zip(rows, new) if 0 <= r < len(self.lens) and 0 < n <= 16 * width]
        need = sum(max(pages_of(n) - pages_of(self.lens[r]), 0) for r, n in do)
        free = self.free()
        if need > len(free):
            return need - len(free)
        for r, n in do:
            for c in range(pages_of(self.lens[r]), pages_of(n)):
                self.table[r, c] = p = free.pop(0)
                self.refs[p] = 1
            self.lens[r] = max(self.lens[r], n)
        return 0

    def fork(self, parents, children):
        rows, before = len(self.lens), self.lens.copy()
        ok = [0 <= p < rows and 0 <= c < rows and self.lens[c] == 0 for p, c in zip(parents, children)]
        free, copies = self.free(), []
        need = sum(bool(o and self.lens[p] % 16) for o, p in zip(ok, parents))
        if need > len(free):
            return need - len(free), [(-1, -1, 0)] * len(parents)
        for o, p, c in zip(ok, parents, children):
            copies.append((-1, -1, 0))
            if not o:
                continue
            n = before[p]
            for i in range(n // 16):
                self.table[c, i] = self.table[p, i]
                self.refs[self.table[p, i]] += 1
            if n % 16:
                self.table[c, n // 16] = q = free.pop(0)
                self.refs[q] = 1
                copies[-1] = (self.table[p, n // 16], q, n % 16)
            self.lens[c] = n
        return 0, copies

    def release(self, rows, keep=None):
        for r, k in zip(rows, keep if keep is not None else [0] * len(rows)):
            if not 0 <= r < len(self.lens):
                continue
            k = max(k, 0)
            for c in range(pages_of(k), pages_of(self.lens[r])):
                self.refs[self.table[r, c]] -= 1
                self.table[r, c] = -1
            self.lens[r] = min(self.lens[r], k)

    def compact(self):
        used = int((self.refs > 0).sum())
        src = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        dst = [p for p in range(used) if self.refs[p] == 0]
        for a, b in zip(src, dst):
            self.refs[b], self.refs[a] = self.refs[a], 0
        to = dict(zip(src, dst))
        for r, n in enumerate(self.lens):
            for c in range(pages_of(n)):
                self.table[r, c] = to.get(self.table[r, c], self.table[r, c])
        return src, dst, used


class Both:
    """A model and a device table that take the same calls."""

    def __init__(self, rows, width, pages, pad=0):
        self.pad = pad  # entries without a row behind every list: what longer lists take is another kernel
        self.m, self.t = Model(rows, width, pages), sp.PageTable.empty(rows, width, pages)
        self.short = dev([-7])
        n = max(sp.sp_pages_workspace_size(pages, 4 * rows + pad), sp.sp_pages_workspace_size(pages, 0))
        self.ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")

    def same(self):
        assert np.array_equal(self.t.ref_counts.cpu().numpy(), self.m.refs)
        assert np.array_equal(self.t.seq_lens.cpu().numpy(), self.m.lens)
        assert np.array_equal(self.t.block_table.cpu().numpy(), self.m.table)
        sp.sp_debug_validate_pages(self.t)

    def reserve(self, rows, new):
        rows, new = [*rows, *[-1] * self.pad], [*new, *[5] * self.pad]
        want = self.m.reserve(rows, new)
        sp.sp_pages_reserve(self.t, dev(rows), dev(new), self.short, self.ws)
        assert int(self.short) == want
        self.same()
        return want

    def fork(self, parents, children):
        parents, children = [*parents, *[-1] * self.pad], [*children, *[0] * self.pad]
        want, copies = self.m.fork(parents, children)
        lists = [dev([-9] * len(parents)) for _ in range(3)]
        sp.sp_pages_fork(self.t, dev(parents), dev(children), *lists, self.short, self.ws)
        assert int(self.short) == want
        assert [tuple(x) for x in torch.stack(lists, 1).tolist()] == copies
        self.same()
        return lists

    def release(self, rows, keep=None):
        self.m.release(rows, keep)
        sp.sp_pages_release(self.t, dev(rows), None if keep is None else dev(keep))
        self.same()

    def compact(self, in_place):
        src, dst, used = self.m.compact()
        table, refs = (self.t.block_table, self.t.ref_counts) if in_place else (torch.full_like(self.t.block_table, -1), torch.full_like(self.t.ref_counts, 99))
        pages = len(self.m.refs)
        a, b, moved = dev([-9] * (pages // 2)), dev([-9] * (pages // 2)), dev([-9, -9])
        sp.sp_pages_compact(self.t, table, refs, a, b, moved, self.ws)
        assert moved.tolist() == [len(src), used]
        n = len(src)
        assert a.tolist() == src + [-9] * (pages // 2 - n) and b.tolist() == dst + [-9] * (pages // 2 - n)
        self.t = sp.PageTable(table, self.t.seq_lens, refs)
        self.same()
        return a, b, moved


@pytest.mark.parametrize("pad", (0, 70), ids=("short-lists", "long-lists"))
@pytest.mark.parametrize("pages", (1, 2, 63, 64, 65, 300, 1023, 1025, 4095, 4096, 4097, 9000, 16383, 16384, 16385))
def test_random_lives(pages, pad):
    rng = np.random.default_rng(pages)
    rows, width = 40, 30
    b = Both(rows, width, pages, pad)
    for step in range(25):
        what = rng.choice(["reserve", "reserve", "fork", "release", "release", "keep", "compact"])
        pick = rng.choice(rows, rng.integers(1, 12), replace=False)
        if what == "reserve":
            b.reserve(pick, rng.integers(0, min(16 * width + 20, 1 + 3 * pages), len(pick)))
        elif what == "fork":
            k = len(pick) // 2 + 1
            parents = rng.choice(pick[:k], 8)
            children = rng.choice(np.setdiff1d(np.arange(rows), pick[:k]), 8, replace=False)
            b.fork(parents, children)
        elif what == "release":
            b.release(pick)
        elif what == "keep":
            b.release(pick, rng.integers(-2, 400, len(pick)))
        else:
            b.compact(in_place=bool(step % 2))


def test_a_pool_larger_than_one_round_of_segments():
    """More than 256 segments of 4096 pages, the free ones scattered over all of them."""
    pages = 4096 * 700 + 77
    b = Both(300, 64, pages)
    rng = np.random.default_rng(1)
    taken = rng.random(pages) < 0.9
    taken[:4096 * 300] = True  # none free in the first round
    b.m.refs[:] = taken
    b.t.ref_counts.copy_(dev(b.m.refs))
    rows, new = np.arange(300), rng.integers(1, 1024, 300)
    free = np.flatnonzero(~taken)
    want, at = np.full((300, 64), -1), 0
    for r, n in zip(rows, new):
        want[r, :pages_of(n)] = free[at:at + pages_of(n)]
        at += pages_of(n)
    sp.sp_pages_reserve(b.t, dev(rows), dev(new), b.short, b.ws)
    assert int(b.short) == 0 and np.array_equal(b.t.block_table.cpu().numpy(), want)
    taken[free[:at]] = True
    assert np.array_equal(b.t.ref_counts.cpu().numpy(), taken.astype(int))
    # and packed together: pages in use that no row holds move too
    a, d, moved = dev([-1] * (pages // 2)), dev([-1] * (pages // 2)), dev([0, 0])
    sp.sp_pages_compact(b.t, b.t.block_table, b.t.ref_counts, a, d, moved, b.ws)
    used = int(taken.sum())
    src, dst = used + np.flatnonzero(taken[used:]), np.flatnonzero(~taken[:used])
    assert moved.tolist() == [len(src), used]
    assert np.array_equal(a.cpu().numpy()[:len(src)], src) and np.array_equal(d.cpu().numpy()[:len(src)], dst)
    to = np.arange(pages)
    to[src] = dst
    assert np.array_equal(b.t.block_table.cpu().numpy(), np.where(want >= 0, to[want], -1))
    assert int(b.t.ref_counts[:used].min()) == 1 and int(b.t.ref_counts[used:].abs().max()) == 0


@pytest.mark.parametrize("pad", (0, 70))
def test_all_or_nothing(pad):
    b = Both(6, 8, 10, pad)
    b.reserve([0, 1], [100, 20])  # 7 + 2 pages: one is left
    assert b.reserve([2, 3], [16, 1]) == 1
    assert b.reserve([2, 3, 4], [128, 128, 128]) == 23
    b.fork([0, 0], [4, 5])  # two partial pages
    b.fork([0], [4])
    b.release([4])
    b.reserve([5], [16])


def test_lists_up_to_the_small_kernel_s_length():
    for n in (1, 15, 16, 17, 33, 63, 64, 65):
        b = Both(140, 40, 6000)
        b.reserve(np.arange(n), 640 - 9 * np.arange(n))
        b.fork(np.arange(n)[::-1], 70 + np.arange(n))
        b.reserve(70 + np.arange(n), [640] * n)
        b.fork([0, 136], [136, 137])  # the second parent is empty when the call is made
        b.compact(in_place=n % 2 == 1)
        b.release(np.arange(140))


@pytest.mark.parametrize("rows,width", [(16, 1024), (128, 128), (1, 3000), (17, 1024), (1, 0), (0, 5)])
def test_compaction_of_small_and_large_tables(rows, width):
    """Up to 16384 entries and pages in one launch."""
    rng = np.random.default_rng(rows)
    for pages in (900, 16384, 16385):
        b = Both(rows, width, pages)
        if rows * width:
            n = min(rows, 12)
            b.reserve(np.arange(n), np.minimum(16 * width, rng.integers(1, 16 * pages // n // 2, n)))
            b.release([0, n // 2], [5, 40])
            b.reserve([n - 1], [16 * min(width, 20)])
            b.release([0])
        b.compact(in_place=pages == 900)
        b.compact(in_place=True)  # nothing left to move


def test_wide_tables():
    for width in (1024, 1025):
        b = Both(9, width, 9000)
        b.reserve([0, 1, 2], [16 * width, 16 * width - 3, 5000])
        b.fork([0, 1, 2], [5, 6, 7])
        b.release([1, 5], [4000, 16 * width - 15])
        b.compact(in_place=True)


def test_lists_longer_than_a_workgroup():
    b = Both(1500, 4, 9000)
    rng = np.random.default_rng(3)
    b.reserve(np.arange(700), rng.integers(1, 65, 700))
    b.fork(rng.integers(0, 700, 800), 700 + np.arange(800))
    b.release(rng.permutation(1500)[:1300], rng.integers(0, 64, 1300))
    b.compact(in_place=False)


@pytest.mark.parametrize("pad", (0, 70))
def test_skipped_entries(pad):
    b = Both(5, 4, 40, pad)
    b.reserve([0, -1, 7, 1, 2], [33, 16, 16, 65, 64])  # rows outside the table, more than a row holds
    b.fork([0, 0, -3, 9, 1, 0], [2, 3, 4, 4, 4, -1])  # a child in use, rows outside, an empty parent
    b.release([-1, 5, 3], [1, 1, 1])


@pytest.mark.parametrize("pad", (0, 70))
def test_the_same_row_twice(pad):
    b, none = Both(4, 8, 64, pad), [-1] * pad
    sp.sp_pages_reserve(b.t, dev([1, 1, 1, *none]), dev([40, 100, 70, *none]), b.short, b.ws)
    sp.sp_debug_validate_pages(b.t)
    assert b.t.seq_lens.tolist() == [0, 100, 0, 0] and int(b.t.ref_counts.sum()) == 7
    sp.sp_pages_reserve(b.t, dev([0]), dev([25]), b.short, b.ws)
    lists = [dev([0, 0, *none]) for _ in range(3)]
    sp.sp_pages_fork(b.t, dev([0, 1, *none]), dev([2, 2, *none]), *lists, b.short, b.ws)  # one of the two
    sp.sp_debug_validate_pages(b.t)
    assert int(b.t.seq_lens[2]) in (25, 100) and sum(x >= 0 for x in lists[0].tolist()) == 1
    sp.sp_pages_release(b.t, dev([1, 1, 1, 2, 2]), dev([50, 20, 90, 0, 0]))
    sp.sp_debug_validate_pages(b.t)
    assert b.t.seq_lens.tolist() == [25, 20, 0, 0] and int(b.t.ref_counts.sum()) == 4


def make_caches(n, pages, heads, d, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda: torch.randint(-32768, 32767, (pages, heads, 16, d), generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)
    return [sp.KVCache(new(), new()) for _ in range(n)]


def copied(pools, src, dst, rows):
    out = [p.view(torch.int16).clone() for p in pools]
    for a, b, r in zip(src, dst, rows):
        if 0 <= a < out[0].shape[0] and 0 <= b < out[0].shape[0]:
            for p, o in zip(pools, out):
                o[b, :, :r] = p.view(torch.int16)[a, :, :r]
    return out


@pytest.mark.parametrize("heads,d", [(1, 64), (1, 128), (2, 64), (3, 64), (8, 128)])
@pytest.mark.parametrize("layers", (1, 3, 70))
def test_copies(heads, d, layers):
    pages = 40 if layers < 10 else 14
    caches = make_caches(layers, pages, heads, d)
    rng = np.random.default_rng(layers)
    perm = rng.permutation(pages)
    n = pages // 2 - 1
    src, dst, rows = perm[:n].copy(), perm[n:2 * n].copy(), rng.integers(0, 17, n)
    src[1], dst[2] = -1, pages  # skipped
    pools = [p for c in caches for p in (c.k_pages, c.v_pages)]
    want = copied(pools, src, dst, rows)
    sp.sp_pages_copy(caches, dev(src), dev(dst), rows=dev(rows))
    for p, w in zip(pools, want):
        assert torch.equal(p.view(torch.int16), w)
    for count in (n + 9, 3, 0, -2):
        want = copied(pools, src[:max(count, 0)], dst, [16] * n)
        sp.sp_pages_copy(caches, dev(src), dev(dst), count=dev([count]))
        for p, w in zip(pools, want):
            assert torch.equal(p.view(torch.int16), w)
    sp.sp_pages_copy(caches[0], dev(src), dev(dst), rows=dev([99] * n), count=dev([n]))


def test_copies_of_many_pages():
    caches = make_caches(2, 30000, 1, 128)
    perm = np.random.default_rng(0).permutation(30000)
    src, dst = torch.from_numpy(perm[:14000]).cuda(), torch.from_numpy(perm[14000:28000]).cuda()
    pools = [p.view(torch.int16) for c in caches for p in (c.k_pages, c.v_pages)]
    want = [p.clone() for p in pools]
    for w in want:
        w[dst] = w[src]
    sp.sp_pages_copy(caches, src.int(), dst.int())
    for p, w in zip(pools, want):
        assert torch.equal(p, w)


def test_a_run_of_them_together():
    """Prompts come in, are sampled several times each, attended, cut back and moved: every row's attention stays that of its tokens."""
    hq, hkv, d, layers = 8, 2, 64, 2
    b = Both(24, 16, 200)
    caches = [sp.KVCache.empty(200, hkv, d, fill_bits=0) for _ in range(layers)]
    g = torch.Generator().manual_seed(5)
    kept = {}  # row -> per layer (K, V) tokens

    def append(rows, counts):
        ctx = [b.m.lens[r] for r in rows]
        b.reserve(rows, [a + n for a, n in zip(ctx, counts)])
        cu, T = dev(np.concatenate([[0], np.cumsum(counts)])), int(sum(counts))
        for layer, cache in enumerate(caches):
            k, v = (torch.randn(T, hkv, d, generator=g).to(torch.bfloat16) for _ in range(2))
            sp.sp_norm_rope_append(cache, None, k.cuda(), v.cuda(), None, cu, dev(ctx), b.t.block_table[dev(rows).long()].contiguous())
            for i, r in enumerate(rows):
                at = int(sum(counts[:i]))
                kk, vv = kept.get((r, layer), (torch.zeros(0, hkv, d), torch.zeros(0, hkv, d)))
                kept[r, layer] = (torch.cat((kk, k[at:at + counts[i]].float())), torch.cat((vv, v[at:at + counts[i]].float())))

    def attend():
        rows = [r for r in range(24) if b.m.lens[r] > 0]
        q = torch.randn(len(rows), hq, d, generator=g).to(torch.bfloat16)
        lens, most = dev(b.m.lens[rows]), int(b.m.lens.max())
        for layer, cache in enumerate(caches):
            out = torch.empty(len(rows), hq, d, dtype=torch.bfloat16, device="cuda")
            n = sp.sp_attn_cross_workspace_size(len(rows), len(rows), 1, most, hq, hkv, d)
            sp.sp_attn_cross(cache, q.cuda(), out, dev(np.arange(len(rows) + 1)), lens, b.t.block_table[dev(rows).long()].contiguous(), 1, most, 0.125,
                             workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))
            for i, r in enumerate(rows):
                k, v = (x.double().repeat_interleave(hq // hkv, dim=1) for x in kept[r, layer])
                assert len(k) == b.m.lens[r]
                w = torch.softmax((k * q[i].double()).sum(-1) * 0.125, dim=0)
                want = (w[..., None] * v).sum(0)
                assert ((out[i].cpu().double() - want).abs() <= 2.0**-8 * want.abs() + 2.0**-7 * (w[..., None] * v.abs()).sum(0)).all()

    append([0, 1, 2, 3], [40, 16, 100, 7])
    parents, children = [0, 0, 1, 2, 2, 3], [4, 5, 6, 7, 8, 9]
    lists = b.fork(parents, children)
    sp.sp_pages_copy(caches, lists[0], lists[1], rows=lists[2])
    for p, c in zip(parents, children):
        for layer in range(layers):
            kept[c, layer] = kept[p, layer]
    attend()
    append([0, 4, 5, 6, 7, 9], [3, 30, 1, 17, 2, 9])
    attend()
    b.release([2, 5])
    b.release([4, 0], [41, 33])  # draft tokens that were not accepted
    for r, n in ((2, 0), (5, 0), (4, 41), (0, 33)):
        for layer in range(layers):
            kept[r, layer] = tuple(x[:n] for x in kept[r, layer])
    attend()
    src, dst, moved = b.compact(in_place=False)
    sp.sp_pages_copy(caches, src, dst, count=moved)
    attend()
    append([4, 8], [9, 20])
    attend()


@pytest.mark.parametrize("pad", (0, 70), ids=("short-lists", "long-lists"))
def test_cut_back_into_a_shared_page(pad):
    """A fork that keeps 20 of its parent's 48 tokens goes on in a row of its own: the parent's pages stay as they are."""
    b = Both(4, 4, 12, pad)
    cache = make_caches(1, 12, 2, 64)[0]
    b.reserve([0], [48])
    b.fork([0], [1])
    b.release([1], [20])
    assert b.m.refs[b.m.table[1, 1]] == 2  # shared, and not full
    bits = cache.k_pages.view(torch.int16)
    before = bits.clone()
    lists = b.fork([1], [2])
    sp.sp_pages_copy(cache, *lists[:2], rows=lists[2])
    b.release([1])
    b.reserve([2], [30])
    own = b.m.table[2, 1]
    assert b.m.refs[own] == 1 and torch.equal(bits[own, :, :4], before[b.m.table[0, 1], :, :4])
    new = torch.ones(10, 2, 64, dtype=torch.bfloat16, device="cuda")
    sp.sp_norm_rope_append(cache, None, new, new, None, dev([0, 10]), dev([20]), b.t.block_table[2:3].contiguous())
    assert (cache.k_pages[own, :, 4:14] == 1).all()
    for page in b.m.table[0, :3]:
        assert torch.equal(bits[page], before[page])


def test_captured():
    """A step that drops, forks, copies and grows, as a graph: every replay against the eager calls on the same table."""
    b = Both(20, 10, 300)
    b.reserve(np.arange(12), 16 + 9 * np.arange(12))
    caches = make_caches(3, 300, 1, 64)
    lists, moves = [dev([0] * 8) for _ in range(3)], [dev([-1] * 150) for _ in range(2)]
    moved, parents, children, new = dev([0, 0]), dev(np.arange(8) % 4), dev(12 + np.arange(8)), dev([120] * 8)
    new_table, new_refs = torch.full_like(b.t.block_table, -1), torch.zeros_like(b.t.ref_counts)

    def step():
        sp.sp_pages_release(b.t, children)
        sp.sp_pages_fork(b.t, parents, children, *lists, b.short, b.ws)
        sp.sp_pages_copy(caches, lists[0], lists[1], rows=lists[2])
        sp.sp_pages_reserve(b.t, children, new, b.short, b.ws)
        sp.sp_pages_compact(b.t, new_table, new_refs, *moves, moved, b.ws)
        sp.sp_pages_copy(caches, *moves, count=moved)

    state = [b.t.block_table, b.t.seq_lens, b.t.ref_counts, *lists, *moves, moved, new_table, new_refs, *[p for c in caches for p in (c.k_pages, c.v_pages)]]
    start = [x.clone() for x in state]
    step()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        parents.copy_(dev(np.random.default_rng(i).integers(0, 12, 8)))
        for x, y in zip(state, start):
            x.copy_(y)
        step()
        want = [x.clone() for x in state]
        for x, y in zip(state, start):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(state, want):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16)) if x.dtype == torch.bfloat16 else torch.equal(x, y)


class Ahead(Both):
    """Rows with room ahead of what is written in them."""

    def __init__(self, rows, width, pages, pad=0):
        super().__init__(rows, width, pages, pad)
        self.written = np.zeros(rows, int)
        self.device = dev(self.written)
        self.t = sp.PageTable(self.t.block_table, self.t.seq_lens, self.t.ref_counts, self.device)

    def fork(self, parents, children):
        self.device.copy_(dev(self.written))
        m, parents, children = self.m, [*parents, *[-1] * self.pad], [*children, *[0] * self.pad]
        tokens = np.minimum(np.maximum(self.written, 0), m.lens)
        ok = [p >= 0 and m.lens[c] == 0 for p, c in zip(parents, children)]
        free, copies = m.free(), []
        need = sum(bool(o and tokens[p] % 16) for o, p in zip(ok, parents))
        want = max(need - len(free), 0)
        for o, p, c in zip(ok, parents, children):
            copies.append((-1, -1, 0))
            if not o or want:
                continue
            n = tokens[p]
            for i in range(n // 16):
                m.table[c, i] = m.table[p, i]
                m.refs[m.table[p, i]] += 1
            if n % 16:
                m.table[c, n // 16] = q = free.pop(0)
                m.refs[q] = 1
                copies[-1] = (m.table[p, n // 16], q, n % 16)
            m.lens[c] = self.written[c] = n
        lists = [dev([-9] * len(parents)) for _ in range(3)]
        sp.sp_pages_fork(self.t, dev(parents), dev(children), *lists, self.short, self.ws)
        assert int(self.short) == want
        assert [tuple(x) for x in torch.stack(lists, 1).tolist()] == copies
        self.same()
        return lists


@pytest.mark.parametrize("pad", (0, 70), ids=("short-lists", "long-lists"))
@pytest.mark.parametrize("pages", (65, 700, 16385))
def test_forks_of_rows_with_room_ahead(pages, pad):
    """A page that is still to be written has one holder, whatever is forked in which order."""
    rng = np.random.default_rng(pages)
    rows, width = 40, 30
    b = Ahead(rows, width, pages, pad)
    for step in range(30):
        pick = rng.choice(rows, rng.integers(2, 12), replace=False)
        what = rng.choice(["reserve", "write", "fork", "fork", "release", "cut"])
        if what == "reserve":
            b.reserve(pick, rng.integers(1, min(16 * width, 2 * pages), len(pick)))
        elif what == "write":
            b.written[pick] += rng.integers(0, b.m.lens[pick] - b.written[pick] + 1)
        elif what == "fork":
            k = len(pick) // 2
            b.fork(rng.choice(pick[:k], 8), rng.choice(np.setdiff1d(np.arange(rows), pick[:k]), 8, replace=False))
        elif what == "release":
            b.written[pick] = 0
            b.release(pick)
        else:
            b.release(pick, b.written[pick] + rng.integers(0, 40, len(pick)))
        for r in range(rows):
            assert (b.m.refs[b.m.table[r, b.written[r] // 16:pages_of(b.m.lens[r])]] == 1).all()


def test_written_lengths_outside_the_room():
    for pad in (0, 70):
        b = Ahead(6, 8, 40, pad)
        b.reserve([0, 1, 2], [100, 40, 16])
        b.written[:3] = [2**31 - 1, -5, 16]  # no more than the room, and none
        b.fork([0, 1, 2], [3, 4, 5])
        assert b.m.lens.tolist() == [100, 40, 16, 100, 0, 16]


@pytest.mark.parametrize("cut", (False, True), ids=("written-lens", "cut-back-first"))
@pytest.mark.parametrize("pad", (0, 70), ids=("short-lists", "long-lists"))
def test_parent_and_child_go_on_in_pages_of_their_own(pad, cut):
    """A row with room for 100 tokens of which 40 are written is forked; both then append, and both keep what they have."""
    pages, hkv, d = 30, 2, 64
    b = Both(3, 8, pages, pad) if cut else Ahead(3, 8, pages, pad)
    cache = make_caches(1, pages, hkv, d)[0]
    tokens = {0: torch.randn(40, hkv, d, device="cuda").to(torch.bfloat16)}

    def append(row, ctx, x):
        sp.sp_norm_rope_append(cache, None, x, x, None, dev([0, len(x)]), dev([ctx]), b.t.block_table[row:row + 1].contiguous())

    b.reserve([0], [100])
    append(0, 0, tokens[0])
    if cut:
        b.release([0], [40])
    else:
        b.written[0] = 40
    lists = b.fork([0], [1])
    sp.sp_pages_copy(cache, lists[0], lists[1], rows=lists[2])
    tokens[1] = tokens[0]
    b.reserve([0, 1], [100, 90])
    for row, n in ((0, 60), (1, 50)):
        new = torch.randn(n, hkv, d, device="cuda").to(torch.bfloat16)
        append(row, 40, new)
        tokens[row] = torch.cat((tokens[row], new))
    for row in (0, 1):
        pos = torch.arange(len(tokens[row]), device="cuda")
        page = b.t.block_table[row].long()[pos // 16]
        for pool in (cache.k_pages, cache.v_pages):
            assert torch.equal(pool[page, :, pos % 16], tokens[row])


@pytest.mark.parametrize("heads,d", [(1, 64), (1, 128), (3, 64)])
def test_more_rows_than_a_page_has(heads, d):
    """Whole pages, and nothing of the page behind."""
    caches, n = make_caches(2, 40, heads, d), 13
    perm = np.random.default_rng(4).permutation(40)
    src, dst, rows = perm[:n], perm[n:2 * n], [99, 16, 17, 2**31 - 1, 15, 0, -1] + [1] * 6
    pools = [p for c in caches for p in (c.k_pages, c.v_pages)]
    want = copied(pools, src, dst, [min(max(r, 0), 16) for r in rows])
    sp.sp_pages_copy(caches, dev(src), dev(dst), rows=dev(rows), count=dev([n]))
    for p, w in zip(pools, want):
        assert torch.equal(p.view(torch.int16), w)
