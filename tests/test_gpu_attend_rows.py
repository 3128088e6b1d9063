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
    """One query vector whose scores rise by hundreds from page to page: what the others get stays bit for bit."""
    c = rising(71, dtype, hd, C, rows, **opts)
    c.call()
    out, lse = bits(c)
    for r, h in ((rows[0] // 2, 1), (0, 6)):
        q = c.q[r, h * hd].clone()
        c.q[r, h * hd] = 100.0 * hd ** 0.5
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
