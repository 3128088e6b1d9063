"""CPU checks of the attention-layer entry points: lsv_rope_init against the oracle's frequencies, and
the refusals of lsv_apply_rope, lsv_append_paged and lsv_attend_paged, all before any HIP call."""
import ctypes
import math

import numpy as np
import pytest

from oracle import attention as OA
from paper_2608_08721_amd import lsv
from tests.test_abi import expect, lib, tiny_cfg  # noqa: F401

BAD = lsv.LSV_ERR_INVALID_ARG
S = 0  # stream handle; never reached


def rope(rot=64, **kw):
    r = lsv.Rope()
    lsv.lsv_rope_init(r, kw.pop("layout", lsv.LSV_ROPE_HALF), rot, kw.pop("base", 10000.0), **kw)
    return r


@pytest.mark.parametrize("rot", [2, 6, 64, 128, 256])
@pytest.mark.parametrize("scaling", range(5))
def test_rope_init_matches_the_oracle(lib, rot, scaling):  # noqa: F811
    if scaling == lsv.LSV_ROPE_NTK and rot == 2:
        expect(BAD, lsv.lsv_rope_init, lsv.Rope(), 0, rot, 10000.0, scaling, 8.0)
        return
    args = dict(factor=8.0, low=1.0, high=4.0, original_ctx=8192)
    r = rope(rot, scaling=scaling, amplitude=1.25, **args)
    want = OA.frequencies(rot, 10000.0, scaling, **args)
    assert (r.layout, r.rot_dim, r.amplitude) == (lsv.LSV_ROPE_HALF, rot, 1.25)
    assert np.allclose(r.freq[:rot // 2], want, rtol=1e-13, atol=0)
    assert not any(r.freq[rot // 2:])


def test_rope_init_refusals(lib):  # noqa: F811
    ok = [0, 64, 10000.0, lsv.LSV_ROPE_BANDS, 8.0, 1.0, 4.0, 8192, 1.0]
    lsv.lsv_rope_init(lsv.Rope(), *ok)
    for i, bad in ((0, 2), (0, -1), (1, 0), (1, 63), (1, 258), (2, 0.0), (2, math.nan), (2, math.inf), (3, 5), (3, -1),
                   (4, 0.0), (4, math.inf), (5, 0.0), (5, 4.0), (6, math.inf), (7, 0), (8, 0.0), (8, math.nan),
                   (8, 1e300)):
        args = list(ok)
        args[i] = bad
        expect(BAD, lsv.lsv_rope_init, lsv.Rope(), *args)
    expect(BAD, lsv.lsv_rope_init, lsv.Rope(), 0, 64, 1.0, lsv.LSV_ROPE_RAMP, 8.0, 1.0, 4.0, 8192, 1.0)
    assert lsv.load().lsv_rope_init(None, 0, 64, 1e4, 0, 1.0, 0.0, 0.0, 0, 1.0) == BAD


def test_apply_rope_refusals(lib):  # noqa: F811
    #       rope, dtype, heads, hd, batch, seq_len, offsets, positions, max_rows, x, xs, y, ys
    ok = [rope(), 1, 4, 64, 2, 16, 16, None, 8, 16, 256, 32, 256, S]
    for i, bad in ((1, 2), (2, 0), (3, 0), (3, 60), (3, 264), (3, 56), (4, 0), (4, 65), (5, None), (6, None), (8, 0),
                   (8, lsv.LSV_MAX_CHUNK_ROWS + 1), (9, None), (10, 255), (11, None), (12, 255)):
        args = list(ok)
        args[i] = bad
        expect(BAD, lsv.lsv_apply_rope, *args)
    in_place = list(ok)
    in_place[11], in_place[12] = in_place[9], 264
    assert "in place" in expect(BAD, lsv.lsv_apply_rope, *in_place)
    for field, bad in (("layout", 3), ("rot_dim", 63), ("rot_dim", 0), ("amplitude", math.inf), ("reserved0", 1.0)):
        r = rope()
        setattr(r, field, bad)
        expect(BAD, lsv.lsv_apply_rope, r, *ok[1:])
    r = rope()
    r.freq[31] = math.nan
    assert "freq[31]" in expect(BAD, lsv.lsv_apply_rope, r, *ok[1:])
    r.freq[31], r.freq[32] = 1.0, math.nan  # behind the rotated pairs: not read (a later refusal shows)
    assert "dtype" in expect(BAD, lsv.lsv_apply_rope, r, 7, *ok[2:])


def test_append_refusals(lib):  # noqa: F811
    cfg = tiny_cfg()
    #      cfg, layer, pool, n_pages, table, max_pages, B, seq, off, positions, max_rows, max_ctx, rope, q.. k.. v..
    ok = [cfg, 1, 16, 9, 16, 4, 2, 16, 16, None, 8, 256, rope(), 16, 256, 32, 256, 48, 256, 64, 256, None, S]
    for i, bad in ((0, tiny_cfg(reserved0=1.0)), (1, -1), (1, 2), (2, None), (2, 8), (3, 0), (4, None), (5, 0),
                   (5, (1 << 20) + 1), (6, 0), (6, 65), (7, None), (8, None), (10, 0), (10, lsv.LSV_MAX_CHUNK_ROWS + 1),
                   (11, 0), (11, 257), (12, rope(128)), (13, None), (15, None), (14, 255), (16, 255), (17, None),
                   (18, 255), (19, None), (20, 255)):
        args = list(ok)
        args[i] = bad
        expect(BAD, lsv.lsv_append_paged, *args)
    expect(lsv.LSV_ERR_UNSUPPORTED, lsv.lsv_append_paged, tiny_cfg(head_dim=96), *ok[1:])


def test_attend_refusals(lib):  # noqa: F811
    cfg = tiny_cfg()
    assert lsv.lsv_attend_workspace_bytes(cfg, 2, 8, 4, 256) > 0
    for bad in ((0, 8, 4, 256), (65, 8, 4, 256), (2, 0, 1, 256), (2, 8, 9, 256), (2, 8, 0, 256), (2, 8, 4, 0)):
        assert lsv.lsv_attend_workspace_bytes(cfg, *bad) == 0
    #      cfg, layer, pool, n_pages, table, max_pages, B, seq, off, max_rows, per_seq, max_ctx, opt, q, out, lse, st, ws
    ok = [cfg, 1, 16, 9, 16, 4, 2, 16, 16, 8, 4, 256, None, 16, 256, 32, 256, None, None, 64, 1 << 30, S]
    for i, bad in ((1, 2), (2, None), (2, 24), (3, 0), (4, None), (5, 0), (6, 65), (7, None), (8, None), (9, 0), (10, 0),
                   (10, 9), (11, 257), (13, None), (13, 24), (14, 252), (14, 257), (15, None), (15, 40), (16, 255),
                   (16, 258), (19, None), (19, 72), (20, 16)):
        args = list(ok)
        args[i] = bad
        expect(BAD, lsv.lsv_attend_paged, *args)
    in_place = list(ok)
    in_place[15], in_place[16] = in_place[13], 260
    expect(BAD, lsv.lsv_attend_paged, *in_place)
    for field, bad in (("scale", math.nan), ("scale", math.inf), ("softcap", -1.0), ("softcap", math.nan),
                       ("softcap", math.inf), ("window", -1), ("reserved0", 1)):
        o = lsv.AttendOptions()
        setattr(o, field, bad)
        expect(BAD, lsv.lsv_attend_paged, *(ok[:12] + [o] + ok[13:]))


def test_attend_workspace_grows_with_every_bound(lib):  # noqa: F811
    """One workspace serves every call of smaller bounds."""
    cfg = tiny_cfg(n_q_heads=32, n_kv_heads=8, head_dim=128, d_model=4096, dtype=lsv.LSV_DTYPE_BF16)
    size = lambda *a: lsv.lsv_attend_workspace_bytes(cfg, *a)  # noqa: E731
    for B in (1, 2, 7, 64):
        for rows in (1, 3, 8, 100, 5000):
            for per in (1, 8, 17, 100, 5000):
                if per > rows:
                    continue
                for ctx in (1, 64, 5000, 200000):
                    here = size(B, rows, per, ctx)
                    assert here > 0
                    assert here <= size(min(64, B + 1), rows, per, ctx)
                    assert here <= size(B, rows + 1, per, ctx)
                    assert here <= size(B, rows + 1, per + 1, ctx)
                    assert here <= size(B, rows, per, ctx + 64)


def test_rows_begin_on_whole_elements(lib):  # noqa: F811
    ok = [rope(), lsv.LSV_DTYPE_BF16, 4, 64, 2, 16, 16, None, 8, 16, 256, 32, 256, S]
    for i in (9, 11):
        expect(BAD, lsv.lsv_apply_rope, *(ok[:i] + [ok[i] + 1] + ok[i + 1:]))
    expect(BAD, lsv.lsv_apply_rope, *(ok[:2] + [65536] + ok[3:]))  # heads
    ok = [tiny_cfg(), 1, 16, 9, 16, 4, 2, 16, 16, None, 8, 256, rope(), 16, 256, 32, 256, 48, 256, 64, 256, None, S]
    for i in (13, 15, 17, 19):  # tiny_cfg is fp32
        expect(BAD, lsv.lsv_append_paged, *(ok[:i] + [ok[i] + 2] + ok[i + 1:]))


def test_attend_refuses_scores_past_fp32(lib):  # noqa: F811
    ok = [tiny_cfg(), 1, 16, 9, 16, 4, 2, 16, 16, 8, 4, 256, None, 16, 256, 32, 256, None, None, 64, 1 << 30, S]
    for field, bad in (("scale", 2e15), ("scale", -2e15), ("softcap", 1e-16), ("softcap", 1e16)):
        o = lsv.AttendOptions()
        setattr(o, field, bad)
        assert "options" in expect(BAD, lsv.lsv_attend_paged, *(ok[:12] + [o] + ok[13:]))


@pytest.mark.parametrize("dtype,tile,heads", [("bf16", 128, 8), ("f32", 32, 1)])
def test_attend_refuses_too_many_pages(lib, dtype, tile, heads):  # noqa: F811
    """One sequence of tiles x pages (x kv heads in the tile kernel) from 2^30 on; one tile fewer is taken
    (a later refusal shows)."""
    cfg = tiny_cfg(n_q_heads=32, n_kv_heads=8, head_dim=128, d_model=4096,
                   dtype=lsv.LSV_DTYPE_BF16 if dtype == "bf16" else lsv.LSV_DTYPE_F32)
    pages, w = 1 << 20, 32 * 128
    tiles = (1 << 30) // (pages * heads)
    for rows, fits in (((tiles - 1) * tile // 4, True), ((tiles - 1) * tile // 4 + 1, False)):
        bounds = (rows, rows, pages * 64)
        assert (lsv.lsv_attend_workspace_bytes(cfg, 1, *bounds) > 0) == fits
        expect(BAD if fits else lsv.LSV_ERR_UNSUPPORTED, lsv.lsv_attend_paged, cfg, 0, 16, 9, 16, pages, 1, 16, 16, *bounds,
               None, 16, w, 32, w, None, None, 64, 0, S)


def test_head_counts_that_no_grid_holds(lib):  # noqa: F811
    many = tiny_cfg(n_q_heads=70000, n_kv_heads=70000, head_dim=64, d_model=64)
    args = [many, 0, 16, 9, 16, 4, 2, 16, 16]
    expect(lsv.LSV_ERR_UNSUPPORTED, lsv.lsv_append_paged, *args, None, 8, 256, None, None, 0, None, 0, 48, 1 << 40, 64, 1 << 40,
           None, S)
    expect(lsv.LSV_ERR_UNSUPPORTED, lsv.lsv_attend_paged, *args, 8, 4, 256, None, 16, 1 << 40, 32, 1 << 40, None, None, 64,
           1 << 40, S)
    one = tiny_cfg(n_q_heads=1024, n_kv_heads=1, head_dim=64, d_model=64)  # 2^30 query vectors of its kv head
    assert lsv.lsv_attend_workspace_bytes(one, 1, 1 << 20, 1 << 20, 64) == 0
    assert lsv.lsv_attend_workspace_bytes(one, 1, (1 << 20) - 1, 1, 64) > 0


def test_tensors_elsewhere_are_refused(lib):  # noqa: F811
    torch = pytest.importorskip("torch")
    host = torch.zeros(64)
    assert "not on the current GPU" in expect(BAD, lsv.lsv_apply_rope, rope(), 1, 4, 64, 2, 16, 16, None, 8, host, 256, 32,
                                              256, S)
    expect(BAD, lsv.lsv_append_paged, tiny_cfg(), 1, 16, 9, host, 4, 2, 16, 16, None, 8, 256, rope(), 16, 256, 32, 256, 48,
           256, 64, 256, None, S)
    expect(BAD, lsv.lsv_attend_paged, tiny_cfg(), 1, 16, 9, 16, 4, 2, 16, 16, 8, 4, 256, None, 16, 256, 32, 256, None, None,
           host, 1 << 30, S)


def test_struct_sizes():
    assert ctypes.sizeof(lsv.Rope) == 16 + 8 * lsv.LSV_ROPE_MAX_DIM // 2
    assert ctypes.sizeof(lsv.AttendOptions) == 40


def test_tensors_of_another_type_or_length_are_refused(lib, monkeypatch):  # noqa: F811
    """The binding's own checks, on tensors that say they lie on the current GPU: none of these calls reaches the library,
    whose refusals (no positions, no rows) show that the right tensors pass."""
    torch = pytest.importorskip("torch")

    class Here(torch.Tensor):
        def get_device(self):
            return 0

    class Driver:
        _cuda_getDevice = staticmethod(lambda: 0)
    monkeypatch.setattr(lsv, "_C", Driver)
    on = lambda *shape, t=torch.int32: torch.zeros(shape, dtype=t).as_subclass(Here)  # noqa: E731
    f32, bf16, u8 = torch.float32, torch.bfloat16, torch.uint8
    cfg, B, P, n_pages = tiny_cfg(), 2, 4, 3  # fp32, 4 heads of 64, two layers
    pool = on(2 * 2 * n_pages * 4 * 64 * 64, t=f32)
    wrong = dict(seq=[on(B, t=torch.int64), on(B - 1), on(2 * B)[::2]], off=[on(B + 1, t=torch.int64), on(B)],
                 table=[on(B, P, t=torch.int64), on(B, P - 1), on(B, P + 1)[:, :P]], status=[on(B, t=f32), on(1)],
                 pool=[on(2, 2, n_pages, 4, 4096, t=bf16), on(2, 2, n_pages - 1, 4, 4096, t=f32),
                       on(pool.nbytes - 1, t=u8), on(2, 2, n_pages, 4, 4096, t=torch.int32)],
                 rows=[on(8, 256, t=bf16), on(8, 256, t=torch.float64)], pos=[on(8, t=torch.int64), on(16)[::2]],
                 lse=[on(8, 4, t=bf16)], ws=[on(64, t=u8)], d_slopes=[on(4, t=torch.float64), on(3, t=f32)],
                 d_key_start=[on(8, t=torch.int64)], d_prefix_len=[on(B, t=torch.int64), on(1)])
    right = dict(seq=on(B), off=on(B + 1), table=on(B, P), status=on(B), pool=pool, rows=on(8, 256, t=f32), pos=on(8),
                 lse=on(8, 4, t=f32), ws=on(1 << 20, t=u8), d_slopes=on(4, t=f32), d_key_start=on(8), d_prefix_len=on(B))

    def rotate(a, dtype=lsv.LSV_DTYPE_F32):
        lsv.lsv_apply_rope(rope(), dtype, 4, 64, B, a["seq"], a["off"], a["pos"], 0, a["rows"], 256, a["rows"],
                           256, S)

    def append(a):
        lsv.lsv_append_paged(cfg, a.get("layer", 1), a["pool"], n_pages, a["table"], P, B, a["seq"], a["off"], a["pos"], 8, 0, rope(),
                             a["rows"], 256, a["rows"], 256, a["rows"], 256, a["rows"], 256, a["status"], S)

    def attend(a):
        o = lsv.AttendOptions(d_slopes=a["d_slopes"])
        o.d_key_start, o.d_prefix_len = a["d_key_start"], a["d_prefix_len"]
        lsv.lsv_attend_paged(cfg, a.get("layer", 1), a["pool"], n_pages, a["table"], P, B, a["seq"], a["off"], 8, 4, 0, o, a["rows"], 256,
                             a["rows"], 256, a["lse"], a["status"], a["ws"], 1 << 20, S)

    for call, names, last in ((rotate, "off pos rows", "max_rows"), (append, "pool table seq off pos rows status", "max_ctx"),
                              (attend, "pool table seq off rows lse status ws d_slopes d_key_start d_prefix_len", "max_ctx")):
        assert last in expect(BAD, call, right)
        assert last in expect(BAD, call, dict(right, pool=on(pool.nbytes, t=u8)))
        assert last in expect(BAD, call, dict(right, pool=on(pool.nbytes // 2, t=u8), layer=0))  # a pool of its own layer
        for name in names.split():
            for x in wrong[name]:
                assert "need a" in expect(BAD, call, dict(right, **{name: x})), (call, name, x.dtype, x.shape)
    # lengths in place of positions, and rows of the other type
    assert "need a" in expect(BAD, rotate, dict(right, pos=None, seq=on(B, t=torch.int64)))
    assert "need a" in expect(BAD, rotate, right, lsv.LSV_DTYPE_BF16)
    assert "max_rows" in expect(BAD, rotate, dict(right, seq=on(1, t=torch.int64)))  # with positions not read


def test_options_keep_their_tensors():
    torch = pytest.importorskip("torch")
    import gc
    import weakref
    o = lsv.AttendOptions(softcap=2.0)
    x = torch.zeros(4)
    o.d_slopes, seen = x, weakref.ref(x)
    at = x.data_ptr()
    del x
    gc.collect()
    assert seen() is not None and o.d_slopes == at and o.softcap == 2.0
    o.d_slopes = at  # an address from now on
    gc.collect()
    assert seen() is None and o.d_slopes == at
    o.d_slopes = ctypes.c_void_p(at)
    assert o.d_slopes == at
    o.d_slopes = None
    assert o.d_slopes is None


def test_frequencies_that_binary64_does_not_hold(lib):  # noqa: F811
    """lsv_rope_init refuses what lsv_apply_rope could not use or would turn into other frequencies, and leaves the
    handle as it was; so does a call with such a handle written by hand."""
    r = lsv.Rope()
    for args in ((0, 64, 1e300, lsv.LSV_ROPE_NTK, 1e9), (0, 64, 1e4, lsv.LSV_ROPE_LINEAR, 1e-309),
                 (0, 64, 1e4, lsv.LSV_ROPE_BANDS, 1e-309, 1.0, 4.0, 8192), (0, 256, 1e-308)):  # (1e-308)^(-254/256) = 4e305
        expect(BAD, lsv.lsv_rope_init, r, *args)
        assert bytes(r) == bytes(ctypes.sizeof(r))
    lsv.lsv_rope_init(r, 0, 64, 1e-290)
    ok = [rope(), 1, 4, 64, 2, 16, 16, None, 8, 16, 256, 32, 256, S]
    ok[0].freq[3] = -1e300
    assert "freq[3]" in expect(BAD, lsv.lsv_apply_rope, *ok)


def test_no_workspace_for_head_counts_that_are_refused(lib):  # noqa: F811
    cfg = lambda n: tiny_cfg(n_q_heads=n, n_kv_heads=n, head_dim=64, d_model=64)  # noqa: E731
    assert lsv.lsv_attend_workspace_bytes(cfg(65536), 2, 8, 4, 256) == 0
    assert lsv.lsv_attend_workspace_bytes(cfg(65535), 2, 8, 4, 256) > 0
