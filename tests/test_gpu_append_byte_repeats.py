"""Appends to the 8-bit cache of rows that share a position, further apart than the 64 rows that a
wave looks at: the last of them is held, whichever token of its block it is."""
import pytest
import torch

from tests.gpu_helpers import DEV
from tests.test_gpu_append_byte import Cache, append
from tests.test_gpu_append import new_rows
from tests.test_gpu_rotary import rope_of

pytestmark = pytest.mark.gpu


def patterns(t):
    """Rows that end with token t more than once: two of them with rows left out in between, a batch
    padded with its last position, a block filled before, and others of its tokens between."""
    b = t - t % 16
    return dict(apart=[t] + [-1] * 63 + [t], further=[t] + [-1] * 70 + [t], much_further=[t] + [-1] * 700 + [t, t],
                padded=[t] * 80, padded_far=[t] * 400, filled=list(range(b, t + 1)) + [t] * 90,
                between=[b, t] + [-1, 10 ** 6] * 40 + [t], thrice=[t] + [-1] * 100 + [t] + [-1] * 100 + [t])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("token", [14, 15])
@pytest.mark.parametrize("name", sorted(patterns(0)))
def test_by_itself(dtype, token, name):
    """The pattern is the whole call: with and without the rows as held, into blocks that keep tokens or none."""
    pos = torch.tensor(patterns(32 + token)[name], dtype=torch.int32)
    _, k, v = new_rows(len(pos), 4, 2, 64, dtype, token)
    c = Cache(1, 200, 4, 2, 64, seed=1)
    append(c, pos, k, v, held=False)
    append(c, pos, k * 3, v)
    append(c, pos, k, v * 9, n_held=torch.tensor([200], dtype=torch.int32))


@pytest.mark.parametrize("token", [14, 15])
@pytest.mark.parametrize("name,before,total",
                         [(n, b, t) for n in sorted(patterns(0)) for b, t in ((0, 300), (30, 700))] +
                         [(n, 3, t) for n in ("apart", "filled", "padded") for t in (2500, 8300)])
def test_among_other_rows(token, name, before, total):
    """The pattern within a sequence and at its end, other rows and sequences around it, in calls of windows
    of 2, 4 and 16 rows and of more than 8,192 rows."""
    rows = list(range(1, 1 + before))
    rows += patterns(32 + token)[name]
    followed = rows + list(range(50, 90))
    r = len(followed)
    n_seqs = max(3, -(-total // r))
    kinds = [followed, rows + [-1] * (r - len(rows)), list(range(r))]
    pos = torch.tensor([kinds[i % 3] for i in range(n_seqs)], dtype=torch.int32).flatten()
    n = len(pos)
    _, k, v = new_rows(n, 2, 1, 64, "bf16", total)
    rope = rope_of(32, 1, 0)
    rp = torch.randint(0, 9000, (1, n), generator=torch.Generator().manual_seed(n), dtype=torch.int32).to(DEV)
    append(Cache(n_seqs, r + 100, 2, 1, 64, seed=2), pos, k, v, rope=rope, rp=rp)
