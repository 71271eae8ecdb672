"""sp_norm_rope_append against its definition in 64 bits: head layouts, rotations, strides, positions, pages, sub-ranges, graphs."""
import numpy as np
import pytest
import torch

import paper_2507_11830_amd as sp

pytestmark = pytest.mark.gpu
CANARY = 0x7FC0


def bf16(gen, *shape, scale=1.5, shift=0.0):
    return (torch.randn(shape, generator=gen) * scale + shift).to(torch.bfloat16)


def angle_table(n, rotary, theta=10000.0):
    at = torch.arange(n, dtype=torch.float64)[:, None] * theta ** -(torch.arange(rotary // 2, dtype=torch.float64) * 2 / rotary)
    return torch.cat([at.cos(), at.sin()], dim=1).float()


def definition(x, weight, eps, cos_sin, interleaved, at):
    """Rows [T, H, d] in 64 bits, and the largest magnitude that goes into a row's rotation."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    most = y.abs().amax(-1, keepdim=True)
    if cos_sin is not None:
        half = cos_sin.shape[1] // 2
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos_sin[at][:, None, :half].double(), cos_sin[at][:, None, half:].double()
        out = y.clone()
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        y = out
    return y, most


def close(got, want, most):
    """One rounding to bf16 (half a step: 2^-8 of the value), and before it at most ten fp32 operations, each off by 2^-24 of the two
    magnitudes that a rotation mixes: 20 x 2^-24 < 2^-19 of the row's largest."""
    got = got.double()
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= 2.0**-8 * want.abs() + 2.0**-19 * most + 1e-38).all()


class Batch:
    def __init__(self, heads, ctx, new, seed, extra_pages=3, packed=True):
        self.hq, self.hkv, self.d = heads
        g = torch.Generator().manual_seed(seed)
        self.ctx, self.new, self.T = np.array(ctx), np.array(new), int(sum(new))
        need = [-(-(a + b) // 16) for a, b in zip(ctx, new)]
        self.num_pages = max(1, sum(need) + extra_pages)
        perm = torch.randperm(self.num_pages, generator=g).numpy().astype(np.int32)
        self.table = np.full((len(new), max(1, max(need))), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = perm[at:at + n]
            at += n
        qkv = bf16(g, self.T, self.hq + 2 * self.hkv, self.d)
        self.q, self.k, self.v = qkv.split((self.hq, self.hkv, self.hkv), dim=1)
        if packed:
            self.dq, self.dk, self.dv = qkv.cuda().split((self.hq, self.hkv, self.hkv), dim=1)
        else:
            self.dq, self.dk, self.dv = (x.contiguous().cuda() for x in (self.q, self.k, self.v))
        self.qw, self.kw = bf16(g, self.d, scale=0.3, shift=1.0), bf16(g, self.d, scale=0.3, shift=1.0)
        self.pos = np.concatenate([np.arange(a, a + b) for a, b in zip(ctx, new)] + [np.zeros(0, int)]).astype(np.int64)
        self.seq = np.repeat(np.arange(len(new)), new)
        self.cache = sp.KVCache.empty(self.num_pages, self.hkv, self.d, fill_bits=CANARY)
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
        self.dctx, self.dtable = torch.tensor(self.ctx, dtype=torch.int32).cuda(), torch.from_numpy(self.table).cuda()
        self.out = torch.full((self.T, self.hq, self.d), float("nan"), dtype=torch.bfloat16, device="cuda")

    def pages(self, keys, rows=None):
        """The pools that the append leaves: K rows (any type), and which of their elements are written."""
        shape = (self.num_pages, self.hkv, 16, self.d)
        k, v, written = torch.zeros(shape, dtype=keys.dtype), torch.zeros(shape, dtype=torch.bfloat16), torch.zeros(shape, dtype=torch.bool)
        for t in range(self.T) if rows is None else rows:
            page, slot = self.table[self.seq[t], self.pos[t] // 16], self.pos[t] % 16
            k[page, :, slot], v[page, :, slot], written[page, :, slot] = keys[t], self.v[t], True
        return k, v, written

    def check(self, qw, kw, eps, cos_sin, interleaved, at=None, rows=None, queries=True):
        at = torch.from_numpy(self.pos if at is None else at)
        keys, most = definition(self.k, kw, eps, cos_sin, interleaved, at)
        k, v, written = self.pages(keys, rows)
        m, _, _ = self.pages(most.expand_as(keys).contiguous(), rows)
        gk, gv = self.cache.k_pages.cpu(), self.cache.v_pages.cpu()
        close(gk[written], k[written], m[written])
        assert torch.equal(gv[written].view(torch.int16), v[written].view(torch.int16))
        for pool in (gk, gv):
            assert (pool.view(torch.int16)[~written] == CANARY).all()
        if queries:
            want, most = definition(self.q, qw, eps, cos_sin, interleaved, at)
            got, keep = self.out.cpu(), np.arange(self.T) if rows is None else np.array(rows)
            close(got[keep], want[keep], most[keep])
            rest = np.setdiff1d(np.arange(self.T), keep)
            assert torch.isnan(got[rest]).all()


SHARDS = [(2, 1, 64), (8, 1, 128), (32, 8, 128), (12, 3, 64), (5, 5, 128), (71, 1, 64), (40, 40, 128)]


@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("norm", (False, True))
@pytest.mark.parametrize("heads,rotary", [(h, r) for h in SHARDS for r in (0, 16, 48, 64, 112, 128) if r <= h[2]], ids=str)
def test_shapes(heads, interleaved, norm, rotary):
    b = Batch(heads, [0, 15, 16, 100, 3], [1, 17, 5, 33, 0], seed=rotary + 3 * norm, packed=rotary % 32 == 0)
    cs = angle_table(160, rotary) if rotary else None
    qw, kw = (b.qw, b.kw) if norm else (None, None)
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable, q_weight=qw.cuda() if norm else None, k_weight=kw.cuda() if norm else None,
                           eps=1e-5, cos_sin=None if cs is None else cs.cuda(), interleaved=interleaved)
    b.check(qw, kw, 1e-5, cs, interleaved)


@pytest.mark.parametrize("batch,new", [(1, 1), (64, 1), (700, 1), (1500, 2), (3, 900), (1, 3000)])
def test_batches(batch, new):
    """Decode batches, ones beyond the staged lengths, long chunks: different lane groups per token."""
    rng = np.random.default_rng(batch)
    b = Batch((8, 1, 128), rng.integers(0, 60, batch), [new] * batch, seed=batch)
    cs = angle_table(4000, 128)
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable, q_weight=b.qw.cuda(), k_weight=b.kw.cuda(), cos_sin=cs.cuda())
    b.check(b.qw, b.kw, 1e-6, cs, False)


def test_one_of_the_norms_and_given_positions():
    for qn, kn in ((True, False), (False, True)):
        b = Batch((16, 2, 64), [5, 0], [20, 7], seed=2)
        at = np.random.default_rng(1).integers(0, 50, b.T)
        cs = angle_table(50, 64)
        sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable, q_weight=b.qw.cuda() if qn else None, k_weight=b.kw.cuda() if kn else None,
                               cos_sin=cs.cuda(), interleaved=True, positions=torch.tensor(at, dtype=torch.int32).cuda())
        b.check(b.qw if qn else None, b.kw if kn else None, 1e-6, cs, True, at=at)


def test_without_norm_and_rotation_it_is_the_append():
    b = Batch((4, 2, 128), [3, 40], [50, 1], seed=3)
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable)
    other = sp.KVCache.empty(b.num_pages, b.hkv, b.d, fill_bits=CANARY)
    sp.sp_kv_append(other, b.dk.contiguous(), b.dv.contiguous(), b.cu, b.dctx, b.dtable)
    for x, y in ((b.cache.k_pages, other.k_pages), (b.cache.v_pages, other.v_pages), (b.out, b.dq.contiguous())):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_keys_and_values_only_and_queries_only():
    b = Batch((8, 2, 64), [0, 9], [30, 12], seed=4)
    cs = angle_table(64, 64)
    sp.sp_norm_rope_append(b.cache, None, b.dk, b.dv, None, b.cu, b.dctx, b.dtable, k_weight=b.kw.cuda(), cos_sin=cs.cuda())
    b.check(None, b.kw, 1e-6, cs, False, queries=False)
    before = [p.clone() for p in (b.cache.k_pages, b.cache.v_pages)]
    sp.sp_norm_rope_append(b.cache, b.dq, None, None, b.out, b.cu, b.dctx, None, q_weight=b.qw.cuda(), cos_sin=cs.cuda())
    b.check(b.qw, b.kw, 1e-6, cs, False)
    for x, y in zip(before, (b.cache.k_pages, b.cache.v_pages)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_in_place_queries():
    b = Batch((33, 1, 128), [7, 1], [40, 90], seed=5, packed=False)
    cs = angle_table(128, 128)
    b.out = b.dq
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.dq, b.cu, b.dctx, b.dtable, q_weight=b.qw.cuda(), k_weight=b.kw.cuda(), cos_sin=cs.cuda())
    b.check(b.qw, b.kw, 1e-6, cs, False)


@pytest.mark.parametrize("shift", (1, 4, 7))
def test_rows_that_begin_anywhere(shift):
    b = Batch((4, 1, 128), [2], [37], seed=6)
    wide = torch.zeros(b.T, 6 * b.d + 13, dtype=torch.bfloat16, device="cuda")
    rows = wide[:, shift:shift + 6 * b.d]
    rows.copy_(torch.cat((b.q, b.k, b.v), dim=1).reshape(b.T, -1).cuda())
    q, k, v = rows.as_strided((b.T, 6, b.d), (wide.stride(0), b.d, 1), shift).split((4, 1, 1), dim=1)
    out = torch.zeros(b.out.numel() + shift, dtype=torch.bfloat16, device="cuda")
    b.out = out[shift:].view(b.out.shape)
    qw = torch.zeros(b.d + shift, dtype=torch.bfloat16, device="cuda")[shift:]
    qw.copy_(b.qw)
    cs = angle_table(64, 96)
    sp.sp_norm_rope_append(b.cache, q, k, v, b.out, b.cu, b.dctx, b.dtable, q_weight=qw, cos_sin=cs.cuda())
    b.check(b.qw, None, 1e-6, cs, False)


def test_sub_range_leaves_the_other_tokens_alone():
    b = Batch((8, 1, 128), [3, 0, 20, 5], [10, 8, 30, 2], seed=7)
    cs = angle_table(64, 128)
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu[1:4], b.dctx[1:3], b.dtable[1:3], q_weight=b.qw.cuda(), k_weight=b.kw.cuda(), cos_sin=cs.cuda())
    b.check(b.qw, b.kw, 1e-6, cs, False, rows=range(10, 48))


def test_bad_pages_and_positions_stay_inside():
    b = Batch((2, 1, 64), [0, 0, 0], [40, 20, 20], seed=8)
    b.dtable[0, 1], b.dtable[1, 0] = -5, b.num_pages + 3  # rows 16..31 of the first sequence, 0..15 of the second
    b.dctx[2] = 10_000_000  # past the block-table row
    cs = angle_table(30, 64)
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable, cos_sin=cs.cuda())
    keep = [t for t in range(60) if not (16 <= t < 32 or 40 <= t < 56)]
    at = np.minimum(b.pos, 29)  # positions past the angles take the last row
    at[60:] = 29
    b.check(None, None, 0, cs, False, at=at, rows=keep, queries=False)
    want, most = definition(b.q, None, 0, cs, False, torch.from_numpy(at))
    close(b.out.cpu(), want, most)


def test_zeros_and_extremes():
    b = Batch((3, 1, 64), [0], [4], seed=9)
    b.dq[0], b.q[0] = 0, 0
    b.dq[1, :, 5], b.dq[2, :, 0] = float("inf"), float("nan")
    one = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable, q_weight=one, eps=1e-6)
    got = b.out.cpu()
    assert (got[0] == 0).all() and torch.isnan(got[1, :, 5]).all() and (got[1, :, :5] == 0).all() and torch.isnan(got[2]).all()
    # an infinity in one row stays out of the others, and where nothing is normalised out of the other pairs of channels
    cs = angle_table(8, 32)
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable, cos_sin=cs.cuda())
    got = b.out.cpu()
    hit = torch.zeros(64, dtype=torch.bool)
    hit[[5, 21]] = True
    assert torch.isfinite(got[1][:, ~hit]).all() and not torch.isfinite(got[1][:, hit]).any() and torch.isfinite(got[3]).all()


def test_empty_calls():
    b = Batch((8, 1, 128), [0], [1], seed=10)
    none = torch.empty(0, 8, 128, dtype=torch.bfloat16, device="cuda")
    kv = torch.empty(0, 1, 128, dtype=torch.bfloat16, device="cuda")
    sp.sp_norm_rope_append(b.cache, none, kv, kv, none.clone(), b.cu, b.dctx, b.dtable)
    assert (b.cache.k_pages.view(torch.int16) == CANARY).all()


def test_captured_with_the_attention_behind_it():
    """The step as it is used: norms, rotation and append, then the decode attention; replays see new rows and lengths."""
    b = Batch((8, 1, 128), [70, 33, 5], [1, 1, 1], seed=11)
    cs, qw, kw = angle_table(256, 128).cuda(), b.qw.cuda(), b.kw.cuda()
    lens = b.dctx + 1
    ws = torch.empty(sp.sp_attn_decode_workspace_size(3, 96, 8, 128), dtype=torch.uint8, device="cuda")
    att = torch.empty_like(b.out)

    def step():
        sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable, q_weight=qw, k_weight=kw, cos_sin=cs)
        sp.sp_attn_decode(b.cache, b.out, att, lens, b.dtable, 96, 0.09, ws)

    b.cache.k_pages.zero_()
    b.cache.v_pages.zero_()
    start = [x.clone() for x in (b.cache.k_pages, b.cache.v_pages)]
    step()
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        b.dq.normal_()
        b.dk.normal_()
        b.dctx.sub_(i)
        lens.sub_(i)
        for x, y in zip((b.cache.k_pages, b.cache.v_pages), start):
            x.copy_(y)
        step()
        want = [x.clone() for x in (b.out, att, b.cache.k_pages, b.cache.v_pages)]
        for x, y in zip((b.cache.k_pages, b.cache.v_pages), start):
            x.copy_(y)
        b.out.fill_(float("nan"))
        att.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((b.out, att, b.cache.k_pages, b.cache.v_pages), want):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_on_another_stream():
    b = Batch((8, 2, 64), [3], [300], seed=12)
    cs = angle_table(400, 64).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sp.sp_norm_rope_append(b.cache, b.dq, b.dk, b.dv, b.out, b.cu, b.dctx, b.dtable, cos_sin=cs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    b.check(None, None, 0, cs.cpu(), False)
