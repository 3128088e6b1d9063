"""What a row gets from lsv_attend_paged does not depend on what it does not see: other rows' queries and keys behind
its position change no bit of it, in any kind of score."""
import numpy as np
import pytest
import torch

from tests.test_gpu_attend import Case
from tests.test_gpu_rope import f64

pytestmark = pytest.mark.gpu


def bits(c):
    torch.cuda.synchronize()
    M = c.s.M
    return c.out[:M, :c.W].clone().view(M, c.s.nq, c.s.hd), c.lse[:M].clone()


def rising(seed, dtype, hd, C, rows, **opts):
    """A case whose keys rise from page to page along dimension 0, which no query looks at."""
    c = Case(seed, 8, 2, hd, dtype, C, rows, **opts)
    s = c.s
    for b in range(s.B):
        n = C[b] + rows[b]
        k, v = c.rng.normal(size=(n, 2, hd)), c.rng.normal(size=(n, 2, hd))
        k[:, :, 0] = (np.arange(n) // 64)[:, None]
        s.write(b, 0, k, v)
    c.q[:s.M, :c.W].view(s.M, 8, hd)[..., 0] = 0.0
    return c


BLOCKS = [([300], [2]), ([300, 70], [40, 90]), ([1000], [64])]
SCORES = [{}, dict(slopes=[0.01] * 8), dict(softcap=30.0), dict(softcap=30.0, slopes=[0.01] * 8)]


@pytest.mark.parametrize("opts", SCORES, ids=lambda o: "-".join(o) or "plain")
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,rows", BLOCKS)
def test_another_rows_scores_change_no_bit(dtype, hd, C, rows, opts):
    """One query vector whose scores rise by hundreds, rise or fall by 1e9 from page to page: what the others get stays bit
    for bit."""
    c = rising(71, dtype, hd, C, rows, **opts)
    c.call()
    out, lse = bits(c)
    for r, h, size in ((rows[0] // 2, 1, 100.0), (0, 6, 100.0), (1, 0, 1e9), (1, 5, -1e9)):
        q = c.q[r, h * hd].clone()
        c.q[r, h * hd] = size * hd ** 0.5
        c.call()
        out1, lse1 = bits(c)
        others = torch.ones(lse.shape, dtype=torch.bool, device="cuda")
        others[r, h] = False
        assert torch.equal(out1[others], out[others]) and torch.equal(lse1[others], lse[others])
        assert not torch.equal(lse1[~others], lse[~others])
        c.q[r, h * hd] = q


@pytest.mark.parametrize("opts", SCORES, ids=lambda o: "-".join(o) or "plain")
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,rows", BLOCKS)
def test_a_key_behind_a_row_changes_no_bit_of_it(dtype, hd, C, rows, opts):
    """A large key at a block's last position: the rows before it, which do not see it, stay bit for bit."""
    c = rising(72, dtype, hd, C, rows, **opts)
    s, last = c.s, C[0] + rows[0] - 1
    c.call()
    out, lse = bits(c)
    k, v = (x[last:last + 1] for x in s.read(0, last + 1))
    q = f64(c.q[rows[0] - 1, :c.W]).reshape(2, 4, hd)[:, 1]
    s.write(0, last, 40.0 * q[None], v)
    c.call()
    out1, lse1 = bits(c)
    before = [r for r in range(s.M) if r != rows[0] - 1]
    assert torch.equal(out1[before], out[before]) and torch.equal(lse1[before], lse[before])
    assert not torch.equal(lse1[rows[0] - 1], lse[rows[0] - 1])


@pytest.mark.parametrize("opts", SCORES, ids=lambda o: "-".join(o) or "plain")
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,rows", BLOCKS)
def test_what_lies_in_unseen_places_changes_no_bit(dtype, C, rows, opts):
    """Places of the pages that hold no key, and keys behind every row's window: NaN, zeros, infinities, large values."""
    c = rising(74, dtype, 128, C, rows, window=90, **opts)
    s, hidden = c.s, C[0] - 89
    empty = torch.isnan(s.pool)
    got = []
    for val in (float("nan"), 0.0, float("inf"), -1e30):
        s.pool[empty] = val
        s.write(0, 0, np.full((hidden, 2, 128), val), np.full((hidden, 2, 128), val))
        c.call()
        got.append(bits(c))
    for out, lse in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1])
    assert torch.isfinite(got[0][0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e3, 1e7, 1e9, 1e12, 1e15, -1e12])
@pytest.mark.parametrize("C,rows", [([700], [2]), ([500, 0], [40, 90]), ([3000], [33])])
def test_scores_far_from_one(dtype, scale, C, rows):
    """Queries and keys of small whole numbers under large scales: a row gets the mean of the values of its best keys,
    equal scores sharing, and log-sum-exp is the best score plus the logarithm of their number.  Scores are exact up to the one
    rounding of the scaled product, the same for equal products; 2^-8 for the rounded probability, 2^-8 the output."""
    c = Case(73, 8, 2, 128, dtype, C, rows, scale=scale)
    s = c.s
    for b in range(s.B):
        n = C[b] + rows[b]
        s.write(b, 0, c.rng.integers(-2, 3, size=(n, 2, 128)), c.rng.normal(size=(n, 2, 128)))
    c.q[:s.M, :c.W] = torch.tensor(c.rng.integers(-2, 3, size=(s.M, c.W)), device="cuda").to(s.t)
    c.call()
    want = c.want()
    out, lse = (f64(x) for x in bits(c))
    n = max(a + r for a, r in zip(C, rows))
    bound = (s.half or 2.0 ** -24) * np.abs(want["out"]) + (s.half + n * 2.0 ** -23) * want["mean_abs"]
    assert np.all(np.abs(out - want["out"]) <= bound)
    assert np.all(np.abs(lse - want["lse"]) <= 2.0 ** -21 * np.abs(want["lse"]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,rows", [([700], [2]), ([500, 300], [40, 90]), ([3000], [33])])
@pytest.mark.parametrize("far", [-2.0 ** 40, -2.0 ** 27, 2.0 ** 40])
def test_scores_that_come_from_far_or_go_there(dtype, C, rows, far):
    """The first 200 keys score `far`, the others as usual: below, they have no share; above, no other key has one."""
    c = Case(75, 8, 2, 128, dtype, C, rows)
    s = c.s
    c.q[:s.M, :c.W].view(s.M, 8, 128)[..., 0] = 1.0
    for b in range(s.B):
        n = C[b] + rows[b]
        k, v = s.read(b, n)
        k[:, :, 0] = np.where(np.arange(n) < 200, far, 0.0)[:, None]
        if far > 0:  # equal scores, exactly
            k[:200, :, 1:] = 0.0
        s.write(b, 0, k, v)
    c.call()
    if far < 0:
        c.opts["key_start"] = [200] * s.M  # of the oracle alone
        c.check()
    else:
        torch.cuda.synchronize()
        mean = np.concatenate([np.repeat(s.read(b, 200)[1].mean(0)[None], rows[b], 0) for b in range(s.B)])
        size = np.concatenate([np.repeat(np.abs(s.read(b, 200)[1]).mean(0)[None], rows[b], 0) for b in range(s.B)])
        out, (mean, size) = f64(bits(c)[0]), (np.repeat(x, 4, axis=1) for x in (mean, size))
        assert np.all(np.abs(out - mean) <= (s.half or 2.0 ** -24) * np.abs(mean) + (s.half + 200 * 2.0 ** -23) * size)
