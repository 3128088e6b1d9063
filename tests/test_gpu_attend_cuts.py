"""lsv_attend_paged in calls that fill the chip: every way in which the tile kernel cuts its units, each checked
against the oracle over all rows.  The cut that the device chose stands in the workspace's first words (pages a split, whole
tiles, parts of each of the rest), so that a case shows that it runs what it is here for."""
import numpy as np
import pytest
import torch

from paper_2608_08721_amd import lsv, runtime
from tests.lsv_testing import i32
from tests.test_gpu_attend import Case
from tests.test_gpu_rope import f64

pytestmark = pytest.mark.gpu
ALL, NONE = 1 << 28, 1 << 30  # no split by length; no tile cut into parts


def cut_of(c):
    torch.cuda.synchronize()
    return c.ws.buf[:12].view(torch.int32).tolist()


def units_of(c):
    s, group = c.s, c.s.nq // c.s.nkv
    return sum(-(-n * group // 128) for n in s.rows) * s.nkv


def twice(c):
    """The call, again with the same bits, and the check against the oracle."""
    c.call()
    how, out, lse = cut_of(c), c.out.clone(), c.lse.clone()
    c.out.fill_(7.0)
    c.lse.fill_(7.0)
    c.call()
    c.check()
    assert torch.equal(c.out, out) and torch.equal(c.lse, lse)
    return how


@pytest.mark.parametrize("nq,nkv,hd,C,rows,opts", [
    (192, 64, 64, [300], [220], {}),                         # 6 tiles of 3 heads a group: 384 units, walks of 5 to 9 pages
    (64, 64, 64, [0, 70], [500, 100], dict(softcap=20.0)),   # 5 tiles, walks from 2 pages on
    (80, 16, 128, [400, 0], [450, 40], dict(window=200))])   # 20 tiles of 5 heads a group: 320 units
def test_one_round_with_its_second_half_turned(nq, nkv, hd, C, rows, opts):
    """More than half a round and no more than one, uncut: long walks stand beside short ones."""
    c = Case(81, nq, nkv, hd, "bf16", C, rows, **opts)
    assert 256 < units_of(c) <= 512
    assert twice(c) == [ALL, NONE, 1]


@pytest.mark.parametrize("nq,nkv,hd,C,rows,opts,whole", [
    (96, 32, 64, [600], [725], {}, 16),                              # 17 tiles: 544 units
    (96, 32, 64, [300, 450, 0], [400, 130, 180], dict(softcap=20.0), 16),
    (48, 16, 128, [500, 640], [900, 530], dict(window=700), 32),     # 35 tiles: 560 units
    (192, 64, 64, [400, 390], [420, 360], {}, 16)])                  # 19 tiles: 1216 units, three of them behind two rounds
def test_a_last_round_in_parts(nq, nkv, hd, C, rows, opts, whole):
    """A few units more than whole rounds hold, with long walks: the tiles of the last round are cut and merged."""
    c = Case(82, nq, nkv, hd, "bf16", C, rows, **opts)
    assert units_of(c) % 512 and units_of(c) > 512
    pps, first, parts = twice(c)
    assert (pps, first) == (ALL, whole) and parts > 1


@pytest.mark.parametrize("nq,nkv,hd,C,rows", [
    (192, 64, 64, [3 * b for b in range(20)], [40 - b % 3 for b in range(20)]),  # 20 tiles of short walks: 1280 units
    (96, 32, 128, [0] * 12, [42 + 40 * (b % 3) for b in range(12)])])            # 24 tiles: 768 units
def test_several_rounds_of_whole_tiles(nq, nkv, hd, C, rows):
    c = Case(83, nq, nkv, hd, "bf16", C, rows)
    assert units_of(c) > 512
    assert twice(c) == [ALL, NONE, 1]


@pytest.mark.parametrize("nq,nkv,hd,C,rows,opts", [
    (24, 8, 128, [4000, 100, 2500], [50, 60, 3], {}), (24, 8, 64, [5000, 0], [30, 41], dict(softcap=20.0, slopes=[0.01] * 24)),
    (6, 2, 128, [9000], [50], dict(key_start=True))])
def test_splits_by_length(nq, nkv, hd, C, rows, opts):
    """Few tiles with long walks: these are split, short sequences' beside them are not."""
    opts = dict(opts)
    if "key_start" in opts:
        opts["key_start"] = [(7 * r) % 9000 for r in range(sum(rows))]
    c = Case(84, nq, nkv, hd, "bf16", C, rows, **opts)
    pps, whole, parts = twice(c)
    assert 4 <= pps < max(C) // 64 and (whole, parts) == (NONE, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,hd,C,rows,opts", [
    (5, 1, 128, [900, 30], [3, 1], {}), (5, 1, 64, [5000], [6], {}), (6, 2, 128, [0, 9000], [7, 2], dict(window=4000)),
    (6, 1, 128, [3000, 10], [90, 44], {}), (5, 1, 64, [40, 700], [160, 33], dict(softcap=20.0)),
    (6, 2, 128, [200, 0], [100, 77], dict(prefix_len=[250, 60])), (96, 32, 64, [600], [725], {})])
def test_in_place(dtype, nq, nkv, hd, C, rows, opts):
    """The output over the queries, whole, split and joined, with groups that straddle tiles: the bits of a call of the
    same bounds with an output of its own."""
    if dtype == "f32" and nkv == 32:
        rows = [100]
    c = Case(85, nq, nkv, hd, dtype, C, rows, **opts)
    c.call()
    c.check()
    queries, lse = c.q.clone(), c.lse.clone()
    for _ in range(3):
        c.q.copy_(queries)
        c.lse.fill_(7.0)
        c.call(out=c.q)
        torch.cuda.synchronize()
        assert torch.equal(c.q[:c.s.M, :c.W], c.out[:c.s.M, :c.W]) and torch.equal(c.lse, lse)
        assert torch.isnan(c.q[c.s.M:]).all()


def test_rows_beside_refused_sequences():
    """Each way to refuse a sequence, in either kernel and type: the others' rows are within the oracle's bounds."""
    for dtype, rows in (("bf16", [2, 9, 1]), ("f32", [2, 9, 1]), ("bf16", [40, 90, 33]), ("f32", [40, 90, 33])):
        C = [100, 50, 30]
        c = Case(86, 8, 2, 128, dtype, C, rows)
        off, n, ctx = [0, rows[0], sum(rows[:2]), sum(rows)], max(rows), max(a + b for a, b in zip(C, rows))
        want = c.want()
        d = 128 * 2.0 ** -24 * want["reach"] + 2.0 ** -22 * (want["reach"] + 1)
        bound = (c.s.half or 2.0 ** -24) * np.abs(want["out"]) + (2 * d[..., None] + c.s.half + ctx * 2.0 ** -23) * want["mean_abs"]
        bad, over = lsv.LSV_ERR_INVALID_ARG, lsv.LSV_ERR_CAPACITY
        for seq, bounds, st in (
                (C, (off[3], n, C[0] + rows[0] - 1), [over, over if C[1] + rows[1] >= C[0] + rows[0] else 0, 0]),
                (C, (off[3], n - 1, ctx), [0, bad, 0]), (C, (off[3] - 1, n, ctx), [0, 0, bad]),
                ([100, -50, 30], (off[3], n, ctx), [0, bad, 0])):
            c.dev = i32(seq), i32(off)
            c.out.fill_(7.0)
            c.call(bounds=bounds, ws=runtime.Workspace(lsv.lsv_attend_workspace_bytes(c.s.cfg, 3, *bounds)))
            torch.cuda.synchronize()
            assert c.s.status.tolist() == st
            for b in range(3):
                mine = slice(off[b], off[b + 1])
                if st[b]:
                    assert (c.out[mine] == 7.0).all()
                else:
                    x = f64(c.out[mine, :c.W]).reshape(-1, 8, 128)
                    assert np.all(np.abs(x - want["out"][mine]) <= bound[mine])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,hd,C,rows,opts", [
    (128, 1, 128, [700, 3], [1, 1], {}), (71, 1, 64, [300, 0, 63], [1, 2, 1], dict(softcap=20.0)),
    (300, 2, 64, [130], [3], dict(window=40)), (33, 1, 128, [5000], [1], {}), (200, 1, 64, [0], [1], {})])
def test_groups_of_more_heads_than_a_tile_holds_rows(dtype, nq, nkv, hd, C, rows, opts):
    """One row's query heads fill tiles, or pass them."""
    c = Case(87, nq, nkv, hd, dtype, C, rows, **opts)
    c.call()
    c.check()


@pytest.mark.parametrize("dtype,nq,nkv", [("bf16", 8, 2), ("f32", 4, 4)])
def test_sixty_four_ragged_sequences(dtype, nq, nkv):
    """The most sequences of a call: empty ones among single tokens and chunks, at the ends too."""
    rows = [0, 1, 40, 3, 0, 70, 2, 1] * 8
    c = Case(88, nq, nkv, 64, dtype, [(37 * b) % 500 for b in range(64)], rows)
    c.call()
    c.check()


def test_one_graph_under_changing_lengths():
    """A call captured once, replayed under lengths for which the device chooses other cuts: whole tiles, a last round in
    parts, splits by length, no rows; eager work between."""
    c = Case(89, 96, 32, 64, "bf16", [600, 700], [725, 300])
    M, per, ctx = c.bounds
    bounds = (M, 725, ctx)
    C, off, seen = i32([0, 0]), i32([0, 0, 0]), set()
    cases = [([600, 700], [725, 300]), ([1300, 60], [25, 30]), ([600, 0], [725, 0]), ([0, 0], [100, 0]), ([5, 5], [0, 0]),
             ([600, 700], [725, 20])]
    c.dev = C, off
    graph = None
    for lens, rows in cases + cases[::-1]:
        C.copy_(i32(lens))
        off.copy_(i32(runtime.row_offsets_of(rows)))
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        c.call(bounds=bounds)
        seen.add(tuple(cut_of(c)))
        want, lse = c.out.clone(), c.lse.clone()
        if graph is None:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                c.call(bounds=bounds)
        for _ in range(3):
            c.out.fill_(7.0)
            c.lse.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert c.s.status.tolist() == [0, 0]
            assert torch.equal(c.out, want) and torch.equal(c.lse, lse)
        assert (want[sum(rows):] == 7.0).all() and (want[:sum(rows), :c.W] != 7.0).any() == (sum(rows) > 0)
    assert len({(pps != ALL, parts > 1) for pps, _, parts in seen}) == 3, seen


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,rows", [([900, 30], [1, 2]), ([300, 0], [60, 33])])
def test_offsets_that_begin_behind_zero(dtype, C, rows):
    """The same rows three places further on: the same bits there, and the rows before them as they were."""
    c = Case(90, 8, 2, 128, dtype, C, rows)
    c.call()
    c.check()
    M, out, lse = c.s.M, c.out[:c.s.M].clone(), c.lse[:c.s.M].clone()
    c.q[3:] = c.q[:M].clone()
    c.q[:3] = float("nan")
    c.dev = i32(C), i32(np.asarray(c.s.off) + 3)
    c.out.fill_(7.0)
    c.lse.fill_(7.0)
    c.call()
    torch.cuda.synchronize()
    assert c.s.status.tolist() == [0, 0]
    assert torch.equal(c.out[3:], out) and torch.equal(c.lse[3:], lse)
    assert (c.out[:3] == 7.0).all() and (c.lse[:3] == 7.0).all()
