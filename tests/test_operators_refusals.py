"""What sp_attn_cross, sp_norm_rope_append and sp_pages_* refuse before anything is launched, and the marshalling of their Python
entry points (no GPU)."""
import ctypes

import pytest

import paper_2507_11830_amd as sp

P = 0x10_0000_0000  # addresses that nothing dereferences
OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, sp.SP_ERR_NULL, sp.SP_ERR_BAD_SHAPE, sp.SP_ERR_UNSUPPORTED, sp.SP_ERR_WORKSPACE


def cache(**kw):
    c = dict(k_pages=P, v_pages=2 * P, num_pages=8, page_size=16, num_kv_heads=2, head_dim=128)
    c.update(kw)
    return sp.sp_cache_desc(*c.values())


def table(**kw):
    t = dict(ref_counts=P, block_table=2 * P, seq_lens=3 * P, num_pages=100, num_rows=4, max_pages_per_seq=9)
    t.update(kw)
    return sp.sp_page_table(*t.values())


def cross(c=None, **kw):
    a = dict(q=P, out=2 * P, cu=3 * P, lens=4 * P, table=5 * P, batch=2, pages=4, total=6, max_q=3, max_kv=40, hq=8, scale=0.1, ws=None, n=0, stream=None)
    a.update(kw)
    return sp.lib().sp_attn_cross(ctypes.byref(c or cache()), *a.values())


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), OK), (dict(total=0), OK), (dict(max_q=0), OK),
    (dict(batch=-1), SHAPE), (dict(total=-1), SHAPE), (dict(pages=-1), SHAPE), (dict(max_q=-1), SHAPE), (dict(max_kv=-1), SHAPE), (dict(pages=0), SHAPE),
    (dict(hq=7), SHAPE), (dict(hq=0), SHAPE), (dict(scale=0.0), UNSUPPORTED), (dict(scale=float("inf")), UNSUPPORTED), (dict(scale=float("nan")), UNSUPPORTED),
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(cu=None), NULL), (dict(lens=None), NULL), (dict(table=None), NULL),
], ids=str)
def test_cross(change, status):
    assert cross(**change) == status


@pytest.mark.parametrize("change,status", [(dict(k_pages=None), NULL), (dict(page_size=32), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(num_pages=0), SHAPE)], ids=str)
def test_descriptors(change, status):
    assert cross(cache(**change)) == status
    assert rope(cache(**change)) == status
    assert sp.lib().sp_pages_copy(ctypes.byref(cache(**change)), 1, P, P, None, None, 3, None) == status


def test_cross_workspace_sizes():
    size = sp.sp_attn_cross_workspace_size
    assert size(0, 5, 5, 100, 8, 1, 128) == 0 and size(1, 5, 5, 100, 7, 2, 128) == 0 and size(1, 5, 5, -1, 8, 1, 128) == 0
    assert size(8, 8 * 4096, 4096, 4096, 8, 1, 128) == 0  # fills the chip
    assert size(1, 40, 40, 9000, 8, 1, 128) >= 2 * 40 * 8 * 130 * 4  # in pieces
    assert size(4, 8, 2, 9000, 8, 1, 128) > 0


def rope(c=None, angles=dict(), **kw):
    a = dict(q=P, k=2 * P, v=3 * P, qs=1024, ks=256, vs=256, out=4 * P, qw=None, kw=None, eps=1e-6)
    b = dict(positions=None, cu=5 * P, ctx=6 * P, table=7 * P, batch=2, pages=4, total=6, hq=8, stream=None)
    for k, v in kw.items():
        (a if k in a else b)[k] = v
    r = dict(cos_sin=8 * P, num_positions=100, rotary_dim=128, interleaved=0)
    desc = None if angles is None else ctypes.byref(sp.sp_rope_desc(*{**r, **angles}.values()))
    return sp.lib().sp_norm_rope_append(ctypes.byref(c or cache()), *a.values(), desc, *b.values())


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), OK), (dict(total=0), OK), (dict(batch=-1), SHAPE), (dict(total=-1), SHAPE), (dict(pages=-1), SHAPE), (dict(hq=-1), SHAPE), (dict(pages=0), SHAPE),
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(cu=None), NULL), (dict(ctx=None), NULL), (dict(table=None), NULL),
    (dict(k=None, v=None, hq=0), NULL),
    (dict(qs=1023), SHAPE), (dict(ks=255), SHAPE), (dict(vs=0), SHAPE), (dict(qs=-1024), SHAPE), (dict(qs=2**62), SHAPE),
    (dict(qw=P, eps=-1e-6), UNSUPPORTED), (dict(kw=P, eps=float("nan")), UNSUPPORTED), (dict(qw=P, eps=float("inf")), UNSUPPORTED),
    (dict(hq=65537, qs=2**24), UNSUPPORTED),
    # q_out over the rows that are read
    (dict(out=P, qs=1536), UNSUPPORTED), (dict(out=P + 2), UNSUPPORTED), (dict(out=P - 2), UNSUPPORTED), (dict(out=P + 6 * 2048 - 2), UNSUPPORTED),
    (dict(out=2 * P), UNSUPPORTED), (dict(out=3 * P + 2 * (5 * 256 + 255)), UNSUPPORTED),
], ids=str)
def test_norm_rope(change, status):
    assert rope(**change) == status


@pytest.mark.parametrize("angles,status", [
    (dict(rotary_dim=8), UNSUPPORTED), (dict(rotary_dim=144), UNSUPPORTED), (dict(rotary_dim=-16), UNSUPPORTED), (dict(interleaved=2), UNSUPPORTED),
    (dict(num_positions=0), SHAPE), (dict(cos_sin=None), NULL)], ids=str)
def test_rotations(angles, status):
    assert rope(angles=angles) == status


def pages_call(name, t=None, n=3, room=None, **null):
    """The call with `room` bytes of workspace, and NULL in the named places."""
    L, t = sp.lib(), t or table()
    size = sp.sp_pages_workspace_size(t.num_pages, 0 if name == "compact" else max(n, 1)) if room is None else room
    g = lambda k: None if k in null else P
    ws = (None if "ws" in null else null.get("at", P), size, None)
    return {
        "reserve": lambda: L.sp_pages_reserve(ctypes.byref(t), g("a"), g("b"), n, g("short"), *ws),
        "fork": lambda: L.sp_pages_fork(ctypes.byref(t), g("a"), g("b"), n, g("src"), g("dst"), g("rows"), g("short"), *ws),
        "release": lambda: L.sp_pages_release(ctypes.byref(t), g("a"), None, n, None),
        "compact": lambda: L.sp_pages_compact(ctypes.byref(t), g("a"), g("b"), g("src"), g("dst"), g("moved"), *ws),
    }[name]()


CALLS = dict(reserve=("a", "b", "short"), fork=("a", "b", "src", "dst", "rows", "short"), release=("a",), compact=("a", "b", "src", "dst", "moved"))


@pytest.mark.parametrize("name", CALLS)
def test_pages(name):
    for place in CALLS[name]:
        assert pages_call(name, **{place: None}) == NULL, place
    for change, status in ((dict(num_pages=0), SHAPE), (dict(num_rows=-1), SHAPE), (dict(max_pages_per_seq=-1), SHAPE), (dict(ref_counts=None), NULL),
                           (dict(block_table=None), NULL), (dict(seq_lens=None), NULL)):
        assert pages_call(name, table(**change)) == status, change
    if name != "compact":
        assert pages_call(name, n=0) == OK and pages_call(name, n=-1) == SHAPE
    if name != "release":
        need = sp.sp_pages_workspace_size(100, 0 if name == "compact" else 3)
        assert need > 0
        assert pages_call(name, room=need - 1) == WORKSPACE and pages_call(name, ws=None) == WORKSPACE and pages_call(name, at=P + 8) == WORKSPACE


def test_copies():
    f = sp.lib().sp_pages_copy
    two = (sp.sp_cache_desc * 2)
    for change in (dict(num_pages=9), dict(num_kv_heads=1), dict(head_dim=64)):
        assert f(two(cache(), cache(**change)), 2, P, P, None, None, 3, None) == SHAPE
    c = ctypes.byref(cache())
    assert f(c, 1, None, P, None, None, 3, None) == NULL and f(c, 1, P, None, None, None, 3, None) == NULL
    assert f(c, 1, P, P, None, None, -1, None) == SHAPE and f(c, -1, P, P, None, None, 1, None) == SHAPE
    assert f(c, 1, None, None, None, None, 0, None) == OK and f(None, 0, P, P, None, None, 3, None) == OK and f(None, 1, P, P, None, None, 3, None) == NULL
    assert f(ctypes.byref(cache(num_kv_heads=65537)), 1, P, P, None, None, 3, None) == UNSUPPORTED
    assert sp.sp_pages_workspace_size(0, 1) == 0 and sp.sp_pages_workspace_size(5, -1) == 0


# ---- marshalling

class T:  # what the binding asks of a tensor
    def __init__(self, ptr, *shape, size=4, strides=None):
        self.ptr, self.shape, self.size, self.strides = ptr, shape, size, strides

    def data_ptr(self):
        return self.ptr

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return self.size

    def stride(self):
        if self.strides:
            return self.strides
        out, n = [], 1
        for s in reversed(self.shape):
            out.insert(0, n)
            n *= s
        return tuple(out)


class Holder:
    def __init__(self, desc):
        self.desc = desc


def plain(x):  # a structure's copy in the place of a pointer to it
    if not isinstance(x, ctypes._Pointer):
        return x
    return type(x.contents).from_buffer_copy(x.contents) if x else None


@pytest.fixture
def seen():
    """The native module bound to functions that note their arguments."""
    sp.lib()
    log, keep, real = [], [], {}
    names = ("sp_kv_append", "sp_attn_prefill", "sp_chunk_step", "sp_attn_decode", "sp_attn_decode_static", "sp_decode_step", "sp_attn_cross",
             "sp_norm_rope_append", "sp_pages_reserve", "sp_pages_fork", "sp_pages_release", "sp_pages_compact", "sp_pages_copy")
    for n in names:
        f = getattr(sp.lib(), n)

        def note(*a, n=n):
            log.append((n, [plain(x) for x in a]))
            return 0

        keep.append(ctypes.CFUNCTYPE(ctypes.c_int, *f.argtypes)(note))
        real[n] = ctypes.cast(keep[-1], ctypes.c_void_p).value
    sp._native.bind(real, ctypes.ArgumentError, ctypes.c_int32, sp.sp_cache_desc, lambda: 0, lambda d: 0x77, lambda: Holder(None), sp.sp_page_table)
    yield log
    sp._bind(sp.lib())


def test_marshalled_arguments(seen):
    c, t = Holder(cache()), Holder(table())
    t.desc.num_rows, ws = 4, T(0x9000, 64, size=1)
    q, out, bt = T(1, 6, 8, 128, size=2), T(2, 6, 8, 128, size=2), T(5, 2, 4)
    sp.sp_attn_cross(c, q, out, T(3, 3), T(4, 2), bt, 3, 40, 0.5, workspace=ws, stream=7)
    name, a = seen.pop()
    assert name == "sp_attn_cross" and a[0].num_pages == 8 and a[1:] == [1, 2, 3, 4, 5, 2, 4, 6, 3, 40, 8, 0.5, 0x9000, 64, 7]
    part = dict(size=2, strides=(12 * 128, 128, 1))
    sp.sp_norm_rope_append(c, T(1, 6, 8, 128, **part), T(11, 6, 2, 128, **part), T(12, 6, 2, 128, **part), out, T(3, 3), T(4, 2), bt, q_weight=T(13, 128, size=2), eps=0.25,
                           cos_sin=T(14, 50, 64), interleaved=True, positions=T(15, 6), stream=7)
    name, a = seen.pop()
    assert name == "sp_norm_rope_append" and a[1:11] == [1, 11, 12, 1536, 1536, 1536, 2, 13, None, 0.25] and a[12:] == [15, 3, 4, 5, 2, 4, 6, 8, 7]
    assert (a[11].cos_sin, a[11].num_positions, a[11].rotary_dim, a[11].interleaved) == (14, 50, 64, 1)
    sp.sp_norm_rope_append(c, None, T(11, 1, 2, 128, size=2, strides=(3, 128, 1)), T(12, 1, 2, 128, size=2), None, T(3, 3), T(4, 2), bt, stream=7)
    name, a = seen.pop()
    assert a[1:10] == [None, 11, 12, 0, 256, 256, None, None, None] and a[10] == pytest.approx(1e-6) and a[11] is None and a[12:] == [None, 3, 4, 5, 2, 4, 1, 0, 7]
    sp.sp_norm_rope_append(c, q, None, None, out, T(3, 3), T(4, 2), None, stream=7)
    name, a = seen.pop()
    assert a[1:8] == [1, None, None, 1024, 0, 0, 2] and a[13:] == [3, 4, None, 2, 0, 6, 8, 7]
    sp.sp_pages_reserve(t, T(1, 3), T(2, 3), T(3, 1), ws, stream=7)
    name, a = seen.pop()
    assert name == "sp_pages_reserve" and a[0].max_pages_per_seq == 9 and a[1:] == [1, 2, 3, 3, 0x9000, 64, 7]
    sp.sp_pages_fork(t, T(1, 3), T(2, 3), T(4, 3), T(5, 3), T(6, 3), T(3, 1), ws, stream=7)
    assert seen.pop()[1][1:] == [1, 2, 3, 4, 5, 6, 3, 0x9000, 64, 7]
    sp.sp_pages_release(t, T(1, 3), T(2, 3), stream=7)
    assert seen.pop()[1][1:] == [1, 2, 3, 7]
    sp.sp_pages_release(t, T(1, 3), stream=7)
    assert seen.pop()[1][1:] == [1, None, 3, 7]
    sp.sp_pages_compact(t, T(1, 4, 9), T(2, 100), T(3, 50), T(4, 50), T(5, 2), ws, stream=7)
    assert seen.pop()[1][1:] == [1, 2, 3, 4, 5, 0x9000, 64, 7]
    sp.sp_pages_copy([c, Holder(cache())], T(1, 3), T(2, 3), rows=T(3, 3), count=T(4, 1), stream=7)
    name, a = seen.pop()
    assert name == "sp_pages_copy" and a[0].head_dim == 128 and a[1:] == [2, 1, 2, 3, 4, 3, 7]
    assert not seen


def test_marshalling_refuses(seen):
    c, t = Holder(cache()), Holder(table())
    q, out, bt, cu, ctx, kv = T(1, 6, 8, 128), T(2, 6, 8, 128), T(5, 2, 4), T(3, 3), T(4, 2), T(9, 6, 2, 128)
    call = lambda *a, **k: sp.sp_norm_rope_append(c, *a, stream=0, **k)
    for bad in (T(1, 6, 8, 64), T(1, 6, 1024), T(1, 5, 8, 128), T(1, 6, 8, 128, strides=(1024, 128, 2)), T(1, 6, 8, 128, strides=(2048, 256, 1))):
        with pytest.raises(ValueError):
            call(bad, kv, kv, out, cu, ctx, bt)
    for bad in (T(2, 6, 4, 128), T(2, 6, 8, 128, strides=(1536, 128, 1))):
        with pytest.raises(ValueError):
            call(q, kv, kv, bad, cu, ctx, bt)
    for k, v in ((T(9, 6, 1, 128), kv), (kv, T(9, 6, 3, 128)), (T(9, 7, 2, 128), T(9, 7, 2, 128))):
        with pytest.raises(ValueError):
            call(q, k, v, out, cu, ctx, bt)
    with pytest.raises(ValueError):
        call(q, kv, kv, out, cu, ctx, T(5, 8))
    with pytest.raises(ValueError):
        call(q, kv, kv, out, cu, ctx, bt, cos_sin=T(1, 50))
    with pytest.raises(ctypes.ArgumentError):
        sp.sp_pages_release(c, T(1, 3), stream=0)  # not a page table
    with pytest.raises(ctypes.ArgumentError):
        sp.sp_pages_copy([t], T(1, 3), T(2, 3), stream=0)  # not a cache
    for args in ((T(1, 3), T(2, 4)), (T(1, 3, 1), T(2, 3))):
        with pytest.raises(ValueError):
            sp.sp_pages_release(t, *args, stream=0)
        with pytest.raises(ValueError):
            sp.sp_pages_reserve(t, *args, T(3, 1), None, stream=0)
        with pytest.raises(ValueError):
            sp.sp_pages_copy([c], *args, stream=0)
    with pytest.raises(ValueError):
        sp.sp_pages_fork(t, T(1, 3), T(2, 3), T(4, 3), T(5, 2), T(6, 3), T(3, 1), None, stream=0)
    for args in ((T(1, 4, 8), T(2, 100), T(3, 50), T(4, 50), T(5, 2)), (T(1, 4, 9), T(2, 99), T(3, 50), T(4, 50), T(5, 2)),
                 (T(1, 4, 9), T(2, 100), T(3, 49), T(4, 50), T(5, 2)), (T(1, 4, 9), T(2, 100), T(3, 50), T(4, 50), T(5, 1))):
        with pytest.raises(ValueError):
            sp.sp_pages_compact(t, *args, None, stream=0)
    assert not seen


def test_no_exception_leaves_the_table_check():
    assert sp.lib().sp_debug_validate_pages(ctypes.byref(table(num_rows=2**31 - 1, max_pages_per_seq=2**31 - 1))) == UNSUPPORTED
    assert sp.lib().sp_debug_validate_pages(None) == NULL and sp.lib().sp_debug_validate_pages(ctypes.byref(table(num_pages=0))) == SHAPE


def test_marshalling_refuses_other_types_and_shapes(seen):
    """Lists of 64-bit numbers (torch's own whole numbers), strided lists, and lists shorter than what is read."""
    c, t = Holder(cache()), Holder(table())
    q, kv, out, bt, cu, ctx = T(1, 6, 8, 128, size=2), T(9, 6, 2, 128, size=2), T(2, 6, 8, 128, size=2), T(5, 2, 4), T(3, 3), T(4, 2)
    good = dict(q=q, k=kv, v=kv, q_out=out, cu_seqlens_new=cu, ctx_lens=ctx, block_table=bt, q_weight=T(13, 128, size=2), k_weight=T(13, 128, size=2), cos_sin=T(14, 50, 64),
                positions=T(15, 6))
    sp.sp_norm_rope_append(c, **good, stream=0)
    sp.sp_norm_rope_append(c, **{**good, "positions": T(15, 9), "cos_sin": T(14, 1, 64, strides=(99, 1))}, stream=0)
    assert len(seen) == 2
    bad = dict(
        cu_seqlens_new=[T(3, 3, size=8)], ctx_lens=[T(4, 2, size=8)],
        block_table=[T(5, 2, 4, size=8)],
        q_weight=[T(13, 127, size=2), T(13, 129, size=2), T(13, 128), T(13, 128, size=2, strides=(2,)), T(13, 1, 128, size=2)],
        k_weight=[T(13, 64, size=2), T(13, 128, size=8), T(13, 128, size=2, strides=(0,))],
        cos_sin=[T(14, 50, 64, size=2), T(14, 50, 64, size=8), T(14, 50, 64, strides=(128, 1)), T(14, 50, 64, strides=(1, 50)), T(14, 50, 64, strides=(64, 2))],
        positions=[T(15, 5), T(15, 6, size=8), T(15, 6, strides=(2,)), T(15, 6, 1)])
    for name, values in bad.items():
        for x in values:
            with pytest.raises(ValueError):
                sp.sp_norm_rope_append(c, **{**good, name: x}, stream=0)
    with pytest.raises(ValueError):
        sp.sp_norm_rope_append(c, None, None, None, None, cu, ctx, bt, stream=0)  # nothing to do it for
    for i, x in enumerate((T(3, 3, size=8), T(4, 2, size=8), T(5, 2, 4, size=8))):
        args = [cu, ctx, bt]
        args[i] = x
        with pytest.raises(ValueError):
            sp.sp_attn_cross(c, q, out, *args, 3, 40, 0.5, stream=0)
    ws, lists, one = T(0x9000, 64, size=1), [T(1, 3), T(2, 3)], T(3, 1)
    for wrong in (T(1, 3, size=8), T(1, 3, size=2), T(1, 3, strides=(2,)), T(1, 3, strides=(0,)), T(1, 2), T(1, 4)):
        for i in range(2):
            args = list(lists)
            args[i] = wrong
            for call in (lambda: sp.sp_pages_reserve(t, *args, one, ws, stream=0), lambda: sp.sp_pages_release(t, *args, stream=0), lambda: sp.sp_pages_copy([c], *args, stream=0)):
                with pytest.raises(ValueError):
                    call()
        for i in range(5):
            args = [T(1, 3) for _ in range(5)]
            args[i] = wrong
            with pytest.raises(ValueError):
                sp.sp_pages_fork(t, *args, one, ws, stream=0)
        with pytest.raises(ValueError):
            sp.sp_pages_copy([c], *lists, rows=wrong, stream=0)
    for wrong in (T(3, 1, size=8), T(3, 0)):
        for call in (lambda: sp.sp_pages_reserve(t, *lists, wrong, ws, stream=0), lambda: sp.sp_pages_fork(t, *[T(1, 3)] * 5, wrong, ws, stream=0),
                     lambda: sp.sp_pages_copy([c], *lists, count=wrong, stream=0)):
            with pytest.raises(ValueError):
                call()
    moves = [T(1, 4, 9), T(2, 100), T(3, 50), T(4, 50), T(5, 2)]
    for i, values in enumerate(((T(1, 4, 9, size=8), T(1, 4, 9, strides=(18, 1)), T(1, 4, 9, strides=(1, 4))), (T(2, 100, size=8),), (T(3, 50, strides=(2,)),), (T(4, 50, size=2),),
                                (T(5, 2, size=8),))):
        for wrong in values:
            args = list(moves)
            args[i] = wrong
            with pytest.raises(ValueError):
                sp.sp_pages_compact(t, *args, ws, stream=0)
    assert len(seen) == 2
    sp.sp_pages_reserve(t, *lists, T(3, size=4), ws, stream=0)  # one counter without dimensions
    sp.sp_pages_compact(t, *moves, ws, stream=0)
    assert len(seen) == 4


@pytest.mark.parametrize("name", CALLS)
def test_more_entries_than_a_launch_holds(name):
    """Refused before the first launch of the call, not by the one that cannot be made."""
    if name == "compact":
        assert pages_call(name, table(num_rows=16000001)) == UNSUPPORTED
    else:
        assert pages_call(name, n=16000001) == UNSUPPORTED and pages_call(name, n=2**31 - 1) == UNSUPPORTED
    assert b"16000000" in sp.lib().sp_last_error()


def test_no_exception_leaves_the_metadata_check():
    assert sp.lib().sp_debug_validate_metadata(ctypes.byref(cache()), P, P, 65536, 2**31 - 1) == UNSUPPORTED
    assert b"memory" in sp.lib().sp_last_error()


def test_marshalling_takes_empty_matrices(seen):
    """Whatever their strides say (torch gives a table of 5 rows and no columns those of one column)."""
    t = Holder(table(max_pages_per_seq=0))
    t.desc.num_rows = 5
    sp.sp_pages_compact(t, T(1, 5, 0, strides=(1, 1)), T(2, 100), T(3, 50), T(4, 50), T(5, 2), T(0x9000, 64, size=1), stream=0)
    q, out = T(1, 6, 8, 128, size=2), T(2, 6, 8, 128, size=2)
    sp.sp_norm_rope_append(Holder(cache()), q, None, None, out, T(3, 3), T(4, 2), None, cos_sin=T(14, 50, 0, strides=(1, 1)), stream=0)
    assert [name for name, _ in seen] == ["sp_pages_compact", "sp_norm_rope_append"] and seen[1][1][11].rotary_dim == 0
