"""sp_attn_cross against its definition in 64 bits: lengths on both sides, head layouts, the kernels behind it, empty encoders,
workspaces, sub-ranges, graphs."""
import math

import numpy as np
import pytest
import torch

import paper_2507_11830_amd as sp
from harness import kernel_launches

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, heads, nq, nk, seed=0, scale=None, spread=1.0, poison=True):
        self.hq, self.hkv, self.d = heads
        self.nq, self.nk = np.array(nq), np.array(nk)
        g = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-int(n) // 16) for n in nk]
        self.num_pages = max(1, sum(need) + 2)
        perm = torch.randperm(self.num_pages, generator=torch.Generator().manual_seed(seed)).numpy().astype(np.int32)
        table = np.full((len(nk), max(1, max(need))), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = perm[at:at + n]
            at += n
        shape = (self.num_pages, self.hkv, 16, self.d)
        k, v = (torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        self.table = torch.from_numpy(table).cuda()
        if poison:  # what lies behind a sequence's last key, and in pages that nobody holds
            there = torch.zeros(self.num_pages, 16, dtype=torch.bool)
            for s, n in enumerate(nk):
                pos = np.arange(n)
                there[table[s, pos // 16], pos % 16] = True
            for p in (k, v):
                p.masked_fill_(~there.cuda()[:, None, :, None], float("nan"))
        self.cache = sp.KVCache(k, v)
        self.T = int(sum(nq))
        self.q = (torch.randn((self.T, self.hq, self.d), generator=g, device="cuda") * spread).to(torch.bfloat16)
        self.out = torch.full_like(self.q, float("nan"))
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(nq)]), dtype=torch.int32).cuda()
        self.lens = torch.tensor(self.nk, dtype=torch.int32).cuda()
        self.scale = 1 / math.sqrt(self.d) if scale is None else scale
        self.max_q, self.max_kv = int(max(nq)), int(max(nk))

    def workspace(self, short=0):
        n = sp.sp_attn_cross_workspace_size(len(self.nq), self.T, self.max_q, self.max_kv, self.hq, self.hkv, self.d)
        return torch.empty(max(n - short, 0), dtype=torch.uint8, device="cuda") if n else None

    def call(self, ws):
        sp.sp_attn_cross(self.cache, self.q, self.out, self.cu, self.lens, self.table, self.max_q, self.max_kv, self.scale, workspace=ws)

    def definition(self, s):
        """(out, sum of weights times |v|) of sequence s in 64 bits."""
        a, b = int(self.cu[s]), int(self.cu[s + 1])
        n, grp = int(self.nk[s]), self.hq // self.hkv
        q = self.q[a:b].double().view(b - a, self.hkv, grp, self.d).permute(1, 2, 0, 3).reshape(self.hkv, -1, self.d)
        pos = torch.arange(n, device="cuda")
        page = self.table[s].long()[pos // 16]
        k, v = (p[page, :, pos % 16].double().permute(1, 0, 2).contiguous() for p in (self.cache.k_pages, self.cache.v_pages))
        w = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()) * self.scale, dim=-1)
        back = lambda x: x.view(self.hkv, grp, b - a, self.d).permute(2, 0, 1, 3).reshape(b - a, self.hq, self.d)
        return back(torch.bmm(w, v)), back(torch.bmm(w, v.abs()))

    def check(self, seqs=None):
        """Half a bf16 step of the output (2^-8), the same of every weight where a row has more than 256 keys (shorter rows take
        their weights as hi + lo), and 2^-13 for fp32 sums of 128 products in the exponent of scores of order ten."""
        got = self.out.double()
        for s in range(len(self.nq)) if seqs is None else seqs:
            a, b = int(self.cu[s]), int(self.cu[s + 1])
            if a == b:
                continue
            x = got[a:b]
            if self.nk[s] == 0:
                assert (x == 0).all(), s
                continue
            want, size = self.definition(s)
            most = 2.0**-8 * want.abs() + (2.0**-13 + (2.0**-8 if self.nk[s] > 256 else 0)) * size
            assert torch.isfinite(x).all(), s
            assert ((x - want).abs() <= most).all(), (s, float(((x - want).abs() - most).max()))


SHARDS = [(2, 1, 64), (8, 1, 128), (32, 8, 128), (12, 3, 64), (16, 2, 64), (5, 5, 128), (12, 2, 128), (64, 1, 128), (7, 1, 64)]


@pytest.mark.parametrize("heads", SHARDS, ids=str)
@pytest.mark.parametrize("nq,nk", [
    ([1, 1, 1, 1], [1, 37, 0, 500]),
    ([3, 0, 4, 1, 2], [16, 90, 64, 0, 700]),
    ([1, 70, 33, 0, 128, 257], [129, 15, 0, 4, 64, 65]),
    ([300, 40], [1, 1000]),
    ([2, 600, 31], [257, 256, 300]),
], ids=("tokens", "few", "mixed", "long-q", "edges"))
def test_lengths_and_heads(heads, nq, nk):
    c = Case(heads, nq, nk, seed=len(nq))
    for ws in (c.workspace(), None):
        c.out.fill_(float("nan"))
        c.call(ws)
        c.check()


@pytest.mark.parametrize("heads", [(8, 1, 128), (16, 2, 64), (32, 8, 128)], ids=str)
@pytest.mark.parametrize("n", (63, 64, 65, 127, 128, 129, 255, 256, 257))
def test_tile_edges(heads, n):
    c = Case(heads, [n, 40, 1], [n, n + 1, n - 1], seed=n)
    c.call(c.workspace())
    c.check()


@pytest.mark.parametrize("heads,nq,nk", [
    ((8, 1, 128), [1] * 64, None),  # equal shares or fixed splits of the decode kernel
    ((8, 1, 128), [1] * 200, None),
    ((16, 2, 64), [4] * 40, None),
    ((4, 1, 128), [16] * 6, None),  # more heads than a column tile holds tokens of
    ((4, 4, 64), [50, 3, 64], [3000, 20, 0]),
    ((8, 1, 128), [1], [30000]),
    ((32, 8, 128), [2, 1], [9000, 5]),
    ((8, 1, 128), [40, 70], [9000, 6000]),  # pieces of the key ranges
    ((16, 2, 64), [100], [12000]),
    ((8, 1, 128), [1000] * 6, [700, 0, 900, 400, 1500, 64]),  # whole tiles
    ((16, 2, 64), [900] * 8, None),  # several workgroups a CU
    ((32, 8, 128), [700, 1200, 30], [333, 2000, 100]),
    ((2, 2, 64), [3000], [3001]),
    ((12, 2, 128), [700, 500, 800], [300, 1, 449]),
    ((5, 5, 128), [1100, 1300, 130, 2000, 7], [511, 257, 256, 270, 640]),
    ((12, 3, 64), [1] * 600, None),  # more sequences than shares are dealt for
], ids=lambda x: "x".join(map(str, x[:3])) if x else "any")
def test_kernels_behind_it(heads, nq, nk):
    rng = np.random.default_rng(len(nq))
    nk = list(rng.integers(1, 2500, len(nq))) if nk is None else nk
    if len(nq) > 30:
        nk[3] = nk[17] = 0
    c = Case(heads, nq, nk, seed=5)
    c.call(c.workspace())
    pick = None if len(nq) < 30 else list(rng.choice(len(nq), 20, replace=False)) + [3, 17]
    c.check(pick)
    first = c.out.clone()
    c.out.fill_(float("nan"))
    c.call(c.workspace())
    assert torch.equal(first.view(torch.int16), c.out.view(torch.int16))  # the same bits again


@pytest.mark.parametrize("heads,nq,nk", [
    ((8, 1, 128), [300, 7, 0, 65], [64, 1, 30, 0]),
    ((8, 1, 128), [5000, 10, 40], [128, 97, 0]),
    ((32, 8, 128), [1500, 33, 600], [256, 129, 31]),  # more than 128 keys: one workgroup a CU
    ((32, 8, 128), [1500, 1400, 1490], [320, 257, 31]),  # of more than 256 keys, and of fewer
    ((12, 3, 64), [200, 500], [32, 33]),
    ((16, 2, 64), [4000, 1], [200, 255]),
    ((7, 1, 64), [50, 3], [33, 100]),
    ((71, 1, 64), [9, 40], [1, 2]),
    ((2, 2, 128), [33, 31, 32], [63, 64, 65]),
    ((64, 1, 128), [300, 2], [16, 17]),
    ((8, 1, 128), [1, 1, 0, 1], [64, 1, 5, 0]),  # few tokens
    ((32, 8, 128), [3, 1] * 20, [100, 7] * 20),
], ids=lambda x: "x".join(map(str, x[:3])))
def test_keys_that_stay_in_lds(heads, nq, nk):
    c = Case(heads, nq, nk, seed=3)
    assert c.workspace() is None
    c.call(None)
    c.check()
    first = c.out.clone()
    grids = kernel_launches(lambda: c.call(None))
    assert len(grids) == 1 and grids[0][1][0] == (256 if max(nk) <= 128 or heads[2] == 64 else 512)
    c.lens.copy_(torch.clamp(c.lens - 1, min=0))  # shorter than the hint says
    c.nk = np.maximum(c.nk - 1, 0)
    c.call(None)
    c.check()
    c.lens += 1000  # and longer: no more than the hint, in memory
    c.call(None)
    assert first.shape == c.out.shape


@pytest.mark.parametrize("heads,nq,nk,launches", [
    ((32, 8, 128), [16, 11, 9, 1], [278, 5, 0, 512], 1),
    ((8, 1, 128), [40, 7, 0, 33], [300, 257, 90, 0], 1),
    ((8, 1, 128), [33], [2000], 2),
    ((16, 2, 64), [30, 1, 64], [900, 0, 600], 2),  # a sequence without states
    ((12, 3, 64), [9, 100, 17], [512, 130, 333], 1),
    ((7, 1, 64), [5, 41, 4], [700, 20, 650], 2),  # four tokens of seven heads a tile
    ((71, 1, 64), [40, 2], [200, 130], 1),  # a head a tile
    ((64, 1, 128), [3, 2], [129, 600], 2),
    ((5, 5, 128), [90, 33, 32, 31], [400, 1, 129, 64], 1),
    ((2, 1, 64), [1000], [777], 2),
    ((8, 1, 128), [8], [60000], 2),
], ids=lambda x: "x".join(map(str, x[:3])) if isinstance(x, (list, tuple)) else str(x))
def test_column_tiles(heads, nq, nk, launches):
    c = Case(heads, nq, nk, seed=13, spread=4.0)
    ws = c.workspace()
    assert launches == 1 or ws is not None
    if ws is not None:
        ws.fill_(0xFF)
    c.call(ws)
    c.check()
    first = c.out.clone()
    grids = kernel_launches(lambda: c.call(ws))
    assert len(grids) == launches and grids[0][1][0] == 256
    c.out.fill_(float("nan"))
    c.call(ws)
    assert torch.equal(first.view(torch.int16), c.out.view(torch.int16))
    c.call(c.workspace(1) if launches == 2 else None)  # less than it takes: another form
    c.check()


@pytest.mark.parametrize("heads,nq,nk", [
    ((32, 8, 128), [500] * 6, [257, 700, 64, 0, 321, 258]),  # also sequences of few keys, and of none
    ((32, 4, 128), [1300, 40, 257, 1], [900, 901, 63, 1]),
    ((8, 1, 128), [2000, 2500], [640, 512]),
    ((12, 2, 128), [1700, 500, 800], [300, 1, 449]),
    ((5, 5, 128), [2100, 1300, 130, 4000, 7], [511, 257, 256, 270, 640]),
    ((64, 1, 128), [300, 2, 333], [400, 577, 16]),
], ids=lambda x: "x".join(map(str, x[:3])))
def test_two_workgroups_a_cu(heads, nq, nk):
    c = Case(heads, nq, nk, seed=11)
    c.call(c.workspace())
    c.check()
    first = c.out.clone()
    grids = kernel_launches(lambda: c.call(c.workspace()))
    assert len(grids) == 1 and grids[0][1][0] == 256
    assert torch.equal(first.view(torch.int16), c.out.view(torch.int16))
    big = Case(heads, nq, nk, seed=12, spread=16.0)  # scores far beyond the first tile's maximum
    big.call(big.workspace())
    big.check()


def test_the_division_of_the_keys_is_taken():
    """Few query tokens on long ranges: pieces and their merge; and with less workspace than asked for, fewer or none."""
    c = Case((8, 1, 128), [40], [9000], seed=1)
    ws = c.workspace()
    c.call(ws)
    grids = kernel_launches(lambda: c.call(ws))
    assert len(grids) == 2 and grids[0][0][2] >= 4
    for short in (1, ws.numel() // 2, ws.numel() - 5):
        c.out.fill_(float("nan"))
        c.call(c.workspace(short))
        c.check()


def test_equals_decode_where_both_apply():
    c = Case((8, 1, 128), [1] * 30, list(range(1, 3001, 100)), seed=2)
    c.call(c.workspace())
    other = torch.empty_like(c.out)
    ws = torch.empty(sp.sp_attn_decode_workspace_size(30, c.max_kv, 8, 128), dtype=torch.uint8, device="cuda")
    sp.sp_attn_decode(c.cache, c.q, other, c.lens, c.table, c.max_kv, c.scale, ws)
    c.check()
    c.out = other
    c.check()


def test_large_scores_and_equal_keys():
    c = Case((8, 1, 128), [130, 5], [700, 90], seed=3, spread=16.0)  # nearly one-hot rows
    c.call(c.workspace())
    c.check()
    c.cache.k_pages.copy_(torch.where(torch.isnan(c.cache.k_pages), c.cache.k_pages, torch.zeros((), dtype=torch.bfloat16, device="cuda")))
    c.call(c.workspace())  # all weights equal: the mean of the values
    c.check()


def test_lengths_beyond_the_table_row_are_cut_there():
    c = Case((8, 1, 128), [20, 3, 200], [64, 32, 64], seed=4)
    c.lens += 1000
    c.nk = np.array([64, 64, 64])
    c.table[1, 2:] = c.table[0, 2:]
    c.cache.k_pages.nan_to_num_(0.0)
    c.cache.v_pages.nan_to_num_(0.0)
    c.max_kv = 64
    for ws in (c.workspace(), None):
        c.call(ws)
        c.check()


def test_no_states_at_all():
    for nq in ([3, 1], [500, 2]):
        c = Case((8, 2, 64), nq, [0, 0], seed=6)
        c.call(c.workspace())
        assert (c.out == 0).all()
        c.out.fill_(float("nan"))
        empty = torch.empty(2, 0, dtype=torch.int32, device="cuda")
        c.lens.fill_(-3)
        sp.sp_attn_cross(c.cache, c.q, c.out, c.cu, c.lens, empty, c.max_q, 0, c.scale)
        assert (c.out == 0).all()


@pytest.mark.parametrize("q,kv", [(1, 3), (3, 1), (20, 1), (1, 20), (50, 50)])
@pytest.mark.parametrize("heads", [(8, 1, 128), (12, 3, 64)], ids=str)
def test_hints_larger_than_the_lengths(heads, q, kv):
    """As of a batch whose buffers are sized for the longest that may come."""
    for nq, nk in (([3, 1, 0, 4], [40, 0, 9, 200]), ([40, 3, 17], [90, 300, 0]), ([300, 200], [100, 500])):
        c = Case(heads, nq, nk, seed=14)
        c.max_q, c.max_kv = c.max_q * q, c.max_kv * kv
        for ws in (c.workspace(), None):
            c.out.fill_(float("nan"))
            c.call(ws)
            c.check()


def test_hints_smaller_than_the_lengths():
    """Rows that are written are right for the states within the hint and any blocks of those behind it, and nothing else is touched."""
    for nq, nk, most_q, most_kv in (([9, 30], [100, 300], 5, 300), ([9, 30], [100, 300], 30, 100), ([400, 90], [700, 600], 90, 700), ([33, 40], [900, 2000], 33, 600)):
        c = Case((8, 1, 128), nq, nk, seed=15)
        c.q = torch.cat((c.q, c.q[:50]))
        c.out = torch.full_like(c.q, float("nan"))
        c.max_q, c.max_kv = most_q, most_kv
        c.call(c.workspace())
        for s, (n, m) in enumerate(zip(nq, nk)):
            a = int(c.cu[s])
            done = min(n, most_q)
            got = c.out[a:a + done].double()
            wants = []
            for keys in {m, min(m, most_kv), *range(-(-most_kv // 32) * 32, m, 32)}:
                c.nk[s] = keys
                wants.append(c.definition(s))
            ok = torch.zeros(done, dtype=torch.bool, device="cuda")
            for want, size in wants:
                ok |= ((got - want[:done]).abs() <= 2.0**-8 * want[:done].abs() + (2.0**-13 + 2.0**-8) * size[:done]).flatten(1).all(1)
            assert ok.all(), (s, nq, nk)
        assert torch.isnan(c.out[sum(nq):]).all()


def test_sub_ranges_and_padded_buffers():
    c = Case((8, 1, 128), [5, 300, 2, 64], [100, 900, 0, 400], seed=7)
    sp.sp_attn_cross(c.cache, c.q, c.out, c.cu[1:4], c.lens[1:3], c.table[1:3], 300, 900, c.scale, workspace=c.workspace())
    c.check([1, 2])
    assert torch.isnan(c.out[:5]).all() and torch.isnan(c.out[307:]).all()
    short = Case((8, 1, 128), [5, 300, 2, 64], [100, 90, 0, 40], seed=17)
    sp.sp_attn_cross(short.cache, short.q, short.out, short.cu[1:4], short.lens[1:3], short.table[1:3], 300, 90, short.scale)
    short.check([1, 2])
    assert torch.isnan(short.out[:5]).all() and torch.isnan(short.out[307:]).all()
    wide = Case((32, 8, 128), [5, 700, 600, 64], [100, 700, 300, 400], seed=18)
    sp.sp_attn_cross(wide.cache, wide.q, wide.out, wide.cu[1:4], wide.lens[1:3], wide.table[1:3], 700, 700, wide.scale)
    wide.check([1, 2])
    assert torch.isnan(wide.out[:5]).all() and torch.isnan(wide.out[1305:]).all()
    few = Case((8, 1, 128), [4, 3, 1, 2], [100, 900, 0, 400], seed=8)
    sp.sp_attn_cross(few.cache, few.q, few.out, few.cu[1:4], few.lens[1:3], few.table[1:3], 4, 900, few.scale, workspace=few.workspace())
    few.check([1, 2])
    assert torch.isnan(few.out[:4]).all() and torch.isnan(few.out[8:]).all()


@pytest.mark.parametrize("most", [20, 128, 300])
def test_more_sequences_than_a_grid_dimension(most):
    """70000 sequences of one query on the same pages, of which each sees another number of states."""
    batch, heads, d = 70000, 2, 64
    c = Case((heads, 1, d), [batch], [most], seed=10, poison=False)
    lens = torch.randint(0, most + 1, (batch,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(10))
    lens[:3] = torch.tensor([0, most, 1])
    table = c.table.expand(batch, -1).contiguous()
    ws = sp.sp_attn_cross_workspace_size(batch, batch, 1, most, heads, 1, d)
    sp.sp_attn_cross(c.cache, c.q, c.out, torch.arange(batch + 1, dtype=torch.int32, device="cuda"), lens.int(), table, 1, most, c.scale,
                     workspace=torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None)
    pos = torch.arange(most, device="cuda")
    k, v = (p[c.table[0].long()[pos // 16], 0, pos % 16].double() for p in (c.cache.k_pages, c.cache.v_pages))
    w = (c.q.double().view(-1, d) @ k.t().contiguous()).view(batch, heads, most) * c.scale
    w = torch.softmax(w.masked_fill(pos[None, None] >= lens[:, None, None], -1e300), -1) * (lens > 0)[:, None, None]
    w = w.view(-1, most)
    got, want, size = c.out.double().view(-1, d), w @ v, w @ v.abs()
    assert ((got - want).abs() <= 2.0**-8 * want.abs() + (2.0**-13 + (2.0**-8 if most > 256 else 0)) * size).all()  # as in Case.check


@pytest.mark.parametrize("nq,nk", [([1] * 8, [900] * 8), ([70, 3], [5000, 200]), ([2000], [1500]), ([400, 30], [90, 60]), ([700] * 6, [500] * 6)], ids=("tokens", "pieces", "tiles", "resident", "two a CU"))
def test_captured(nq, nk):
    c = Case((8, 1, 128), nq, nk, seed=9)
    ws = c.workspace()
    c.call(ws)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            c.call(ws)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        c.q.normal_()
        c.lens.sub_(7 * i)
        c.call(ws)
        want = c.out.clone()
        c.out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(want.view(torch.int16), c.out.view(torch.int16))


def test_pages_beyond_four_gigabytes():
    """A pool whose last pages lie past 32-bit byte offsets, for the calls that write and read it."""
    heads, pages = 8, 140_000  # 4.6 GB each for K and V
    cache = sp.KVCache(*(torch.empty(pages, heads, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    g = torch.Generator(device="cuda").manual_seed(1)
    nk, nq = [70, 33], [5, 40]
    far = torch.tensor([[pages - 1, pages - 7, pages - 3, pages - 2, pages - 9], [pages - 20, 3, pages - 21, -1, -1]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[0, 1, 2, 4, 5], [6, 7, 8, -1, -1]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(103, heads, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    cu_k, zero = torch.tensor([0, 70, 103], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    sp.sp_norm_rope_append(cache, None, k, v, None, cu_k, zero, far)
    for pool, x in ((cache.k_pages, k), (cache.v_pages, v)):
        assert torch.equal(pool[pages - 9, :, 5].view(torch.int16), x[69].view(torch.int16))
    q = torch.randn(45, 8, 128, generator=g, device="cuda").to(torch.bfloat16)
    cu, lens = torch.tensor([0, 5, 45], dtype=torch.int32, device="cuda"), torch.tensor(nk, dtype=torch.int32, device="cuda")
    src, dst = far.flatten()[[0, 1, 2, 3, 4, 5, 7]], near.flatten()[[0, 1, 2, 3, 4, 5, 7]]
    sp.sp_pages_copy(cache, src, dst)
    near[1, 1] = 3
    outs = []
    for table in (far, near):
        outs.append(torch.empty_like(q))
        sp.sp_attn_cross(cache, q, outs[-1], cu, lens, table, 40, 70, 0.09)
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16)) and torch.isfinite(outs[0]).all()
    sp.sp_pages_copy(cache, dst, src)  # and back over the boundary
    sp.sp_attn_cross(cache, q, outs[1], cu, lens, far, 40, 70, 0.09)
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
    # the other kernels, which the hint for the keys selects
    many = torch.randn(4500, 8, 128, generator=g, device="cuda").to(torch.bfloat16)
    chunks = torch.tensor([0, 500, 4500], dtype=torch.int32, device="cuda")
    for x, ends, longest, most in ((q, cu, 40, 400), (q[:9], torch.tensor([0, 5, 9], dtype=torch.int32, device="cuda"), 5, 400), (many, chunks, 4000, 300), (many, chunks, 4000, 4000)):
        got = []
        for table in (far, near):
            got.append(torch.full_like(x, float("nan")))
            sp.sp_attn_cross(cache, x, got[-1], ends, lens, table, longest, most, 0.09)
        assert torch.equal(got[0].view(torch.int16), got[1].view(torch.int16)) and torch.isfinite(got[0]).all()


EVERY_KEY = [
    ((8, 1, 128), [1], [30000]),  # shares and their merge
    ((32, 8, 128), [2, 1], [9000, 5]),
    ((12, 3, 64), [1] * 600, "uneven"),  # more sequences than shares are dealt for
    ((8, 1, 128), [1] * 64, "uneven"),  # splits of the longest range
    ((16, 2, 64), [4] * 32, "uneven"),
    ((8, 1, 128), [40, 70], [9000, 6000]),  # pieces
    ((16, 2, 64), [100], [12000]),
    ((8, 1, 128), [8], [60000]),  # column tiles
    ((12, 3, 64), [9, 100, 17], [512, 130, 333]),
    ((8, 1, 128), [5000, 10, 40], [128, 97, 0]),  # keys that stay in LDS
    ((32, 8, 128), [1500, 1400, 1490], [320, 257, 31]),
    ((8, 1, 128), [2000, 2500], [640, 512]),  # two workgroups a CU
    ((12, 3, 64), [600, 17, 300], [2500, 65, 700]),  # halves
    ((8, 1, 128), [1000] * 6, [1700, 0, 1900, 400, 1500, 64]),  # whole tiles
]


@pytest.mark.parametrize("edges", (False, True), ids=("blocks", "first-and-last-of-32"))
@pytest.mark.parametrize("heads,nq,nk", EVERY_KEY, ids=lambda x: "x".join(map(str, x[:3])) if isinstance(x, (list, tuple)) else str(x))
def test_every_block_of_keys_counts_once(heads, nq, nk, edges):
    """All scores are 0, so all weights are 1, which bf16 holds.  A block of 32 keys (or the first and the last key of one) has values of 1 in one channel,
    the next block in the next, and so on: a block that is lost, or taken twice, moves its channel by 1 / (blocks of that channel), asserted to be
    several times the only rounding there is, half a bf16 step (2^-8)."""
    nk = [int(x) for x in np.random.default_rng(3).integers(100, 2000, len(nq))] if nk == "uneven" else nk
    if len(nq) > 30:
        nk[3] = nk[17] = 0
    c = Case(heads, nq, nk, seed=21)
    k, v = c.cache.k_pages, c.cache.v_pages
    for p in (k, v):
        p.copy_(torch.where(torch.isnan(p), p, torch.zeros((), dtype=p.dtype, device="cuda")))
    wants = []
    for s, n in enumerate(nk):
        pos = torch.arange(n, device="cuda")
        item = pos // 32
        if edges:
            chosen = (pos % 32 == 0) | (pos % 32 == 31) | (pos == n - 1)
            pos, item = pos[chosen], torch.arange(int(chosen.sum()), device="cuda")
        page = c.table[s].long()[pos // 16]
        want = torch.zeros(c.hkv, c.d, dtype=torch.float64, device="cuda")
        items = torch.zeros(c.d, device="cuda").index_add_(0, torch.unique(item) % c.d, torch.ones(len(torch.unique(item)), device="cuda"))
        assert items.max() <= 2**5  # one of them is 2^-5 of the channel, eight times the rounding
        for h in range(c.hkv):
            channel = (item + 7 * h) % c.d
            v[page, h, pos % 16, channel] = 1
            want[h].index_add_(0, channel, torch.full((len(pos),), 1 / max(n, 1), dtype=torch.float64, device="cuda"))
        wants.append(want.repeat_interleave(c.hq // c.hkv, dim=0))
    for ws in (c.workspace(), None):
        c.out.fill_(float("nan"))
        c.call(ws)
        for s in range(len(nk)):
            got = c.out[int(c.cu[s]):int(c.cu[s + 1])].double()
            assert ((got - wants[s]).abs() <= (2.0**-8 + 2.0**-20) * wants[s]).all(), s


@pytest.mark.parametrize("spread", (4.0, 16.0))
@pytest.mark.parametrize("heads,nq,nk", [
    ((8, 1, 128), [300, 7, 0, 65], [64, 33, 30, 0]), ((8, 1, 128), [5000, 10, 40], [128, 97, 0]), ((32, 8, 128), [1500, 33, 600], [256, 129, 31]),
    ((32, 8, 128), [1500, 1400, 1490], [320, 257, 31]), ((16, 2, 64), [4000, 1], [200, 255]), ((7, 1, 64), [50, 3], [33, 100]), ((32, 8, 128), [3, 1] * 20, [100, 7] * 20),
], ids=lambda x: "x".join(map(str, x[:3])))
def test_scores_far_beyond_the_first_block_s_in_lds(heads, nq, nk, spread):
    """Keys that stay in LDS, rows whose maximum moves from block to block.  A score is a sum of d products in fp32, off by at most d * 2^-24 of
    the sum of their magnitudes (A); its weight by that times the scale, the output by twice that of sum(w |v|).  Weights as hi + lo: 2^-16, or bf16 (2^-8)
    beyond 256 keys; fp32 sums of up to 320 of them: 2^-15.  Half a bf16 step of the output: 2^-8."""
    c = Case(heads, nq, nk, seed=22, spread=spread)
    assert c.workspace() is None
    c.call(None)
    for s in range(len(nk)):
        a, b = int(c.cu[s]), int(c.cu[s + 1])
        if a == b or nk[s] == 0:
            assert (c.out[a:b] == 0).all()
            continue
        want, size = c.definition(s)
        pos = torch.arange(nk[s], device="cuda")
        keys = c.cache.k_pages[c.table[s].long()[pos // 16], :, pos % 16].double().abs()  # [keys, KV heads, d]
        rows = c.q[a:b].double().abs().view(b - a, c.hkv, -1, c.d)
        most = max(float((rows[:, h].reshape(-1, c.d) @ keys[:, h].t().contiguous()).max()) for h in range(c.hkv))
        off = 2 * c.d * 2.0**-24 * most * c.scale + 2.0**-15 + (2.0**-8 if nk[s] > 256 else 2.0**-16)
        got = c.out[a:b].double()
        assert torch.isfinite(got).all() and ((got - want).abs() <= 2.0**-8 * want.abs() + off * size).all(), s


def test_more_keys_than_the_hint_in_lds():
    """Sequences longer than the hint that sizes the LDS: any number of states between the hint and the length, none behind the table's row."""
    for heads, nq, nk in (((8, 1, 128), [300, 7, 65], [64, 10, 33]), ((32, 8, 128), [1500, 33, 600], [256, 129, 31]), ((16, 2, 64), [4000, 1], [200, 255]), ((7, 1, 64), [50, 3], [33, 100])):
        c = Case(heads, nq, nk, seed=23)
        for p in (c.cache.k_pages, c.cache.v_pages):
            p.nan_to_num_(0.25)
        c.table.clamp_(min=0)
        hint, width = c.max_kv, 16 * c.table.shape[1]
        c.lens += 1000
        c.call(None)
        for s, n in enumerate(nq):
            got, ok = c.out[int(c.cu[s]):int(c.cu[s + 1])].double(), None
            for keys in range(min(hint, width), width + 1):
                c.nk[s] = keys
                want, size = c.definition(s)
                fits = ((got - want).abs() <= 2.0**-8 * want.abs() + (2.0**-13 + 2.0**-8) * size).flatten(1).all(1)
                ok = fits if ok is None else ok | fits
            assert ok.all(), s
