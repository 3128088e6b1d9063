"""lsv_apply_rope and lsv_append_paged against the oracle.

Bounds.  A cosine or sine is off by the rounding of the reduced angle (1/2 turn of 2^-24, times pi:
2^-23.3) and two units of sincospi (2^-23); with the amplitude's and the products' and sum's roundings
(five of 2^-24) a rotated element is within (|a| + |b|) * amplitude * 2^-21 before it is stored, and
storing in bf16 adds 2^-8 of the value (2^-24 in fp32, inside the bound above).  Copied elements, V and
everything that the call does not name are bit for bit what they were."""
import numpy as np
import pytest
import torch

from oracle import attention as OA
from paper_2608_08721_amd import lsv, runtime
from tests.lsv_testing import i32
from tests.test_ops_abi import rope as make_rope

pytestmark = pytest.mark.gpu
DT = {"bf16": (torch.bfloat16, lsv.LSV_DTYPE_BF16, 2.0 ** -8), "f32": (torch.float32, lsv.LSV_DTYPE_F32, 0.0)}


def rows_of(rng, M, width, pad, dtype, shift=0):
    """[M, width] values in rows width + pad elements apart, `shift` elements off the allocation; the gaps hold NaN."""
    buf = torch.full((shift + M * (width + pad) + 8,), float("nan"), dtype=dtype, device="cuda")
    view = buf[shift:shift + M * (width + pad)].view(M, width + pad)
    view[:, :width] = torch.tensor(rng.normal(size=(M, width)), device="cuda").to(dtype)
    return buf, view


def f64(t):
    return t.double().cpu().numpy()


def check_rotated(got, x, pos, freq, layout, amp, half_step):
    want = OA.rope(x, pos, freq, layout, amp)
    rot = 2 * len(freq)
    size = np.abs(x[..., :rot])
    pair = size[..., :rot // 2] + size[..., rot // 2:] if layout == OA.HALF else size[..., 0::2] + size[..., 1::2]
    both = np.concatenate([pair, pair], -1) if layout == OA.HALF else np.repeat(pair, 2, axis=-1)
    bound = both * abs(amp) * 2.0 ** -21 + half_step * np.abs(want[..., :rot])
    assert np.all(np.abs(got[..., :rot] - want[..., :rot]) <= bound)
    assert np.array_equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [OA.HALF, OA.INTERLEAVED])
@pytest.mark.parametrize("heads,hd,rot,M,pad,shift", [
    (1, 8, 2, 1, 0, 0), (3, 64, 64, 17, 0, 0), (40, 128, 128, 33, 256, 0), (5, 128, 32, 700, 16, 0),
    (2, 256, 256, 9, 0, 0), (3, 80, 32, 5, 0, 0), (2, 64, 12, 7, 0, 0), (3, 64, 64, 6, 3, 1), (4, 128, 64, 3, 1, 5)])
def test_rope_positions(dtype, layout, heads, hd, rot, M, pad, shift):
    t, code, half = DT[dtype]
    rng = np.random.default_rng(M + rot)
    pos = rng.integers(-5, 200000, size=M)
    pos[0] = 0
    r = make_rope(rot, layout=layout, amplitude=1.25)
    W = heads * hd
    _, x = rows_of(rng, M, W, pad, t, shift)
    out, y = rows_of(rng, M + 2, W, pad, t, shift)
    before = out.clone()
    x0 = x.clone()
    lsv.lsv_apply_rope(r, code, heads, hd, 1, None, i32([0, M]), i32(pos), M + 2, x, W + pad, y, W + pad)
    torch.cuda.synchronize()
    got, freq = f64(y[:M, :W]).reshape(M, heads, hd), np.array(r.freq[:rot // 2])
    check_rotated(got, f64(x0[:, :W]).reshape(M, heads, hd), pos, freq, layout, 1.25, half)
    # the gaps, and the rows past the last one, are left alone
    after, named = out.clone(), torch.zeros_like(out, dtype=torch.bool)
    named[shift:shift + M * (W + pad)].view(M, W + pad)[:, :W] = True
    assert torch.equal(after[~named].view(torch.uint8), before[~named].view(torch.uint8))
    # in place, without row offsets: the same bits
    lsv.lsv_apply_rope(r, code, heads, hd, 1, None, None, i32(pos), M, x, W + pad, x, W + pad)
    torch.cuda.synchronize()
    assert torch.equal(x[:, :W], y[:M, :W])
    if pad:
        assert torch.isnan(x[:, W:]).all()


def test_rope_positions_from_the_lengths():
    """Without d_positions a row sits at its sequence's length plus its index: empty sequences, 64 of them."""
    rng = np.random.default_rng(0)
    for rows in ([3, 0, 1, 70], [0, 0, 5], list(rng.integers(0, 4, size=64))):
        C = rng.integers(0, 5000, size=len(rows))
        off = runtime.row_offsets_of(rows)
        M = int(off[-1])
        pos = np.concatenate([C[b] + np.arange(n) for b, n in enumerate(rows)])
        x = torch.tensor(rng.normal(size=(M, 128)), device="cuda", dtype=torch.float32)
        y = [torch.zeros_like(x) for _ in range(2)]
        r = make_rope(64)
        lsv.lsv_apply_rope(r, lsv.LSV_DTYPE_F32, 2, 64, len(rows), i32(C), i32(off), None, M + 9, x, 128, y[0], 128)
        lsv.lsv_apply_rope(r, lsv.LSV_DTYPE_F32, 2, 64, len(rows), None, i32(off), i32(pos), M, x, 128, y[1], 128)
        torch.cuda.synchronize()
        assert torch.equal(y[0], y[1]) and y[0].abs().sum() > 0


def test_rope_leaves_rows_alone_under_a_bad_last_offset():
    x = torch.ones((8, 64), device="cuda")
    for last in (-1, 9):
        lsv.lsv_apply_rope(make_rope(), lsv.LSV_DTYPE_F32, 1, 64, 1, i32([3]), i32([0, last]), None, 8, x, 64, x, 64)
    torch.cuda.synchronize()
    assert torch.equal(x, torch.ones_like(x))


class Layer:
    """One layer's pool of a small model with scattered pages: everything that is not written holds NaN
    (bf16 and fp32 alike), table entries behind a sequence's pages are outside the pool."""

    def __init__(self, rng, nq, nkv, hd, dtype, C, rows, layers=1, layer=0, spare=2):
        self.t, self.code, self.half = DT[dtype]
        self.nq, self.nkv, self.hd, self.C, self.rows, self.layer = nq, nkv, hd, list(C), list(rows), layer
        self.B, self.off = len(C), runtime.row_offsets_of(rows)
        self.M = int(self.off[-1])
        self.cfg = lsv.ModelConfig(n_layers=layers, d_model=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=hd, d_ff=4, vocab=1,
                                   dtype=self.code, rms_eps=1e-5, reserved0=0.0, rope_base=1e4)
        pages = [-(-(c + n) // 64) for c, n in zip(C, rows)]
        self.max_pages, self.n_pages = max(pages) + 1, sum(pages) + spare
        self.table_np = np.full((self.B, self.max_pages), -1, dtype=np.int32)
        order = rng.permutation(self.n_pages)
        at = 0
        for b, n in enumerate(pages):
            self.table_np[b, :n] = order[at:at + n]
            at += n
        self.table = i32(self.table_np)
        self.pool = torch.full((layers, 2, self.n_pages, nkv, 64 * hd), float("nan"), dtype=self.t, device="cuda")
        self.max_ctx = max(1, max(c + n for c, n in zip(C, rows)))
        self.status = torch.full((self.B,), 99, dtype=torch.int32, device="cuda")

    def places(self, b, pos):
        """Flat indices into the layer's pool (K, V) of positions pos of sequence b: [len(pos), nkv, hd]."""
        pos = np.asarray(pos)
        page = self.table_np[b, pos // 64].astype(np.int64)[:, None, None]
        h, d, j = np.arange(self.nkv)[None, :, None], np.arange(self.hd)[None, None, :], (pos % 64)[:, None, None]
        block = (page * self.nkv + h) * 64 * self.hd
        return block + j * self.hd + d, self.n_pages * self.nkv * 64 * self.hd + block + d * 64 + runtime.v_column(j)

    def write(self, b, start, k, v):
        flat = self.pool[self.layer].view(-1)
        for at, x in zip(self.places(b, np.arange(start, start + len(k))), (k, v)):
            flat[torch.tensor(at, device="cuda")] = torch.tensor(x, device="cuda").to(self.t)

    def read(self, b, n):
        flat = self.pool[self.layer].view(-1)
        return [f64(flat[torch.tensor(at, device="cuda")]) for at in self.places(b, np.arange(n))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,hd,rot,layout,C,rows,pad", [
    (4, 4, 64, 64, OA.HALF, [0], [1], 0), (8, 2, 128, 128, OA.HALF, [63, 5, 64], [1, 0, 2], 0),
    (8, 2, 128, 64, OA.INTERLEAVED, [1531], [257], 64), (6, 2, 64, 32, OA.HALF, [0, 130, 60], [200, 64, 9], 0),
    (3, 1, 128, 128, OA.INTERLEAVED, [10, 20], [128, 1], 8), (4, 2, 64, 24, OA.HALF, [62], [5], 3),
    (32, 8, 128, 128, OA.HALF, list(range(0, 640, 10)), [1] * 64, 0)])
def test_append(dtype, nq, nkv, hd, rot, layout, C, rows, pad):
    rng = np.random.default_rng(sum(C) + rot)
    s = Layer(rng, nq, nkv, hd, dtype, C, rows, layers=2, layer=1)
    W = (nq + 2 * nkv) * hd
    buf, x = rows_of(rng, s.M + 3, W, pad, s.t, 0)
    x[s.M:] = float("nan")
    q_out = torch.full((s.M + 3, nq * hd), 7.0, dtype=s.t, device="cuda")
    r = make_rope(rot, layout=layout, amplitude=0.75)
    before = s.pool.clone()
    call = lambda rope, pos, q, qs, qo, qos: lsv.lsv_append_paged(  # noqa: E731
        s.cfg, 1, s.pool, s.n_pages, s.table, s.max_pages, s.B, i32(C), i32(s.off), pos, s.M + 3, s.max_ctx, rope, q, qs,
        qo, qos, x[:, nq * hd:], W + pad, x[:, (nq + nkv) * hd:], W + pad, s.status)
    call(r, None, x, W + pad, q_out, nq * hd)
    torch.cuda.synchronize()
    assert s.status.tolist() == [0] * s.B
    heads = f64(x[:s.M, :W]).reshape(s.M, nq + 2 * nkv, hd)
    pos = np.concatenate([c + np.arange(n) for c, n in zip(C, rows)])
    freq = np.array(r.freq[:rot // 2])
    check_rotated(f64(q_out[:s.M]).reshape(s.M, nq, hd), heads[:, :nq], pos, freq, layout, 0.75, s.half)
    assert (q_out[s.M:] == 7.0).all()
    named = torch.zeros(s.pool[0].numel(), dtype=torch.bool, device="cuda")
    flat = s.pool[1].view(-1)
    for b in range(s.B):
        mine = slice(s.off[b], s.off[b + 1])
        kat, vat = (torch.tensor(a, device="cuda") for a in s.places(b, C[b] + np.arange(rows[b])))
        check_rotated(f64(flat[kat]), heads[mine, nq:nq + nkv], pos[mine], freq, layout, 0.75, s.half)
        assert np.array_equal(f64(flat[vat]), heads[mine, nq + nkv:])
        named[kat.reshape(-1)] = True
        named[vat.reshape(-1)] = True
    assert torch.equal(flat[~named].view(torch.uint8), before[1].view(-1)[~named].view(torch.uint8))
    assert torch.equal(s.pool[0].view(torch.uint8), before[0].view(torch.uint8))
    # again with the positions given, queries in place: the same bits; without a rotation: copies; without queries
    once = s.pool.clone()
    lsv.lsv_append_paged(s.cfg, 1, s.pool, s.n_pages, s.table, s.max_pages, s.B, i32(C), i32(s.off),
                         i32(np.append(pos, [0, 0, 0])), s.M + 3, s.max_ctx, r, x, W + pad, x, W + pad, x[:, nq * hd:],
                         W + pad, x[:, (nq + nkv) * hd:], W + pad, None)
    torch.cuda.synchronize()
    assert torch.equal(s.pool.view(torch.uint8), once.view(torch.uint8))
    assert torch.equal(x[:s.M, :nq * hd], q_out[:s.M])
    call(None, None, None, 0, None, 0)
    torch.cuda.synchronize()
    for b in range(s.B):
        kat, vat = (torch.tensor(a, device="cuda") for a in s.places(b, C[b] + np.arange(rows[b])))
        assert np.array_equal(f64(flat[kat]), heads[s.off[b]:s.off[b + 1], nq:nq + nkv])
        assert np.array_equal(f64(flat[vat]), heads[s.off[b]:s.off[b + 1], nq + nkv:])


def test_append_statuses_and_pages_outside_the_pool():
    """Refused sequences and pages outside the pool are not written; their neighbours are."""
    rng = np.random.default_rng(9)
    C, rows = [10, 100, 20, 0], [3, 70, 4, 5]
    s = Layer(rng, 2, 2, 64, "f32", C, rows)
    W = 6 * 64
    x = torch.tensor(rng.normal(size=(s.M, W)), device="cuda", dtype=s.t)

    def call(lengths, off, max_rows, max_ctx):
        s.pool.fill_(float("nan"))
        q_out = torch.full((s.M, 128), 7.0, device="cuda")
        lsv.lsv_append_paged(s.cfg, 0, s.pool, s.n_pages, s.table, s.max_pages, s.B, i32(lengths), i32(off), None,
                             max_rows, max_ctx, None, x, W, q_out, 128, x[:, 128:], W, x[:, 256:], W, s.status)
        torch.cuda.synchronize()
        flat = s.pool.view(-1)
        wrote = [int(torch.isfinite(flat[torch.tensor(s.places(b, C[b] + np.arange(rows[b]))[0], device="cuda")]).all())
                 for b in range(s.B)]
        return s.status.tolist(), wrote, q_out, int(torch.isfinite(flat).sum())

    st, wrote, q_out, n = call(C, s.off, s.M, 169)  # sequence 1 ends at 170
    assert (st, wrote) == ([0, lsv.LSV_ERR_CAPACITY, 0, 0], [1, 0, 1, 1])
    assert (q_out[3:73] == 7.0).all() and (q_out[:3] == x[:3, :128]).all()
    st, wrote, _, _ = call([10, 100, -1, 0], s.off, s.M, 256)
    assert (st, wrote) == ([0, 0, -1, 0], [1, 1, 0, 1])
    st, wrote, _, _ = call(C, s.off, s.M - 1, 256)  # the last sequence runs past max_rows
    assert (st, wrote) == ([0, 0, 0, -1], [1, 1, 1, 0])
    st, _, _, n = call(C, [0, 5, 3, 4, 6], s.M, 256)  # decreasing, then behind an earlier offset: rows 3.. are sequence 0's
    assert st == [0, -1, -1, -1] and n == 2 * 5 * 128
    s.table[1, 2] = s.n_pages  # positions 128..169 of sequence 1 have no page
    st, wrote, q_out, n = call(C, s.off, s.M, 256)
    assert st == [0] * 4 and wrote == [1, 0, 1, 1] and n == 2 * (s.M - 42) * 128 and (q_out != 7.0).all()


def test_rope_at_the_largest_bounds():
    """As many rows and heads as a call takes."""
    r = make_rope(8)
    for M, heads in ((lsv.LSV_MAX_CHUNK_ROWS, 1), (3, 65535)):
        x = torch.randn((M, heads * 8), device="cuda")
        y = torch.zeros_like(x)
        lsv.lsv_apply_rope(r, lsv.LSV_DTYPE_F32, heads, 8, 1, i32([5]), i32([0, M]), None, M, x, heads * 8, y, heads * 8)
        torch.cuda.synchronize()
        rows = np.unique(np.append(np.arange(0, M, 65521), M - 1))
        check_rotated(f64(y)[rows].reshape(len(rows), heads, 8), f64(x)[rows].reshape(len(rows), heads, 8), 5 + rows,
                      np.array(r.freq[:4]), OA.HALF, 1.0, 0.0)


def test_rope_and_append_on_another_stream():
    rng = np.random.default_rng(12)
    s = Layer(rng, 4, 2, 64, "bf16", [60, 3], [9, 1])
    x = torch.tensor(rng.normal(size=(10, 8 * 64)), device="cuda").to(s.t)
    y, q = torch.zeros_like(x), torch.zeros((10, 256), dtype=s.t, device="cuda")
    r = make_rope(64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lens, off = i32([60, 3]), i32([0, 9, 10])
    torch.cuda.synchronize()
    lsv.lsv_apply_rope(r, lsv.LSV_DTYPE_BF16, 6, 64, 2, lens, off, None, 10, x, 512, y, 512, side)
    lsv.lsv_append_paged(s.cfg, 0, s.pool, s.n_pages, s.table, s.max_pages, 2, lens, off, None, 10, s.max_ctx, r, x, 512, q,
                         256, x[:, 256:], 512, x[:, 384:], 512, s.status, side.cuda_stream)
    side.synchronize()
    assert s.status.tolist() == [0, 0] and torch.equal(q, y[:, :256])
    k = np.concatenate([s.read(b, c + n)[0][c:] for b, (c, n) in enumerate(((60, 9), (3, 1)))])
    assert np.array_equal(k.reshape(10, 128), f64(y[:, 256:384]))


@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("dtype,rot,M", [("bf16", 64, 40), ("f32", 64, 40), ("bf16", 12, 700), ("f32", 64, 3000)])
def test_rope_takes_the_rows_that_the_offsets_name(dtype, rot, M, positions):
    """Offsets that begin behind 0: the rows before the first are as they were, in place too."""
    t, code, half = DT[dtype]
    rng = np.random.default_rng(5)
    x = torch.tensor(rng.normal(size=(M + 5, 128)), device="cuda").to(t)
    r, first = make_rope(rot), M // 3
    C, off = [11, 500, 7], [first, first + 4, first + 4, M]
    seq = i32(C)
    whole = np.concatenate([np.full(first, 3), 11 + np.arange(4), 7 + np.arange(M - first - 4)])
    want = x.clone()
    lsv.lsv_apply_rope(r, code, 2, 64, 1, None, None, i32(whole), M, x, 128, want, 128)
    want[:first] = x[:first]
    y = x.clone()
    args = (None, i32(off), i32(whole)) if positions else (seq, i32(off), None)
    lsv.lsv_apply_rope(r, code, 2, 64, 3, *args, M + 5, y, 128, y, 128)
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_rope_leaves_refused_sequences_alone():
    """Offsets and lengths that the append refuses: those rows stay as they were, the others turn."""
    r = make_rope()
    x = torch.tensor(np.random.default_rng(6).normal(size=(12, 64)), device="cuda").float()

    def turned(pos):
        y = x.clone()
        lsv.lsv_apply_rope(r, lsv.LSV_DTYPE_F32, 1, 64, 1, None, None, i32(pos), 12, x, 64, y, 64)
        return y
    for C, off, rows in (([5, -1, 9], [0, 2, 7, 12], {0: (0, 2), 2: (7, 12)}),     # a negative length
                         ([5, 6, 9], [0, 9, 3, 12], {0: (0, 9)}),                  # decreasing, then behind an earlier offset
                         ([5, 2 ** 31 - 3, 9], [0, 2, 7, 12], {0: (0, 2), 2: (7, 12)}),  # positions past 32 bits
                         ([5, 6, 9], [-1, 2, 7, 12], {}), ([5, 6, 9], [13, 2, 7, 12], {}), ([5, 6, 9], [0, 2, 7, 13], {})):
        want = x.clone()
        for b, (a, z) in rows.items():
            want[a:z] = turned(C[b] + np.arange(12) - a)[a:z]
        y = x.clone()
        lsv.lsv_apply_rope(r, lsv.LSV_DTYPE_F32, 1, 64, 3, i32(C), i32(off), None, 12, y, 64, y, 64)
        torch.cuda.synchronize()
        assert torch.equal(y, want), (C, off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_takes_the_rows_that_the_offsets_name(dtype):
    """Offsets that begin behind 0: the pages and queries of a call without the rows before them."""
    rng = np.random.default_rng(13)
    C, rows, first = [61, 0], [70, 3], 5
    s = Layer(rng, 4, 2, 64, dtype, C, rows)
    x = torch.tensor(rng.normal(size=(s.M + first, 8 * 64)), device="cuda").to(s.t)
    r, got = make_rope(64), []
    for at in (0, first):
        s.pool.fill_(float("nan"))
        q = torch.full((s.M + first, 256), 7.0, dtype=s.t, device="cuda")
        rows_ = x[first - at:]
        lsv.lsv_append_paged(s.cfg, 0, s.pool, s.n_pages, s.table, s.max_pages, 2, i32(C), i32(s.off + at), None, s.M + at,
                             s.max_ctx, r, rows_, 512, q, 256, rows_[:, 256:], 512, rows_[:, 384:], 512, s.status)
        torch.cuda.synchronize()
        assert s.status.tolist() == [0, 0] and (q[:at] == 7.0).all()
        got.append((q[at:at + s.M].clone(), s.pool.clone().view(torch.uint8)))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
