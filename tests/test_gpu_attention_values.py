"""NaN and infinities in cached values: every row that sees the token has them in the elements that hold them, no other
row and no other element has anything of them.  The keys stay finite, so that only the values can carry them."""
import numpy as np
import pytest
import torch

from gpu_util import say
from test_gpu_attention import BF, F8, FP, HALF, TINY, U, Case, tk  # noqa: F401

pytestmark = pytest.mark.gpu
STEP = 5                                                               # spoil k takes the elements d with d % STEP == k


def _spoil(c, spoils, junk):
    """spoils: (request, position, k).  Returns which elements [token][dim] see one."""
    bad = np.zeros((c.total, c.value), dtype=bool)
    for r, p, k in spoils:
        page = int(c.tables[r, p // c.page])
        values = c.pool[page, c.planes - 1, p % c.page].to(torch.float32)
        values[:, k::STEP] = junk
        c.pool[page, c.planes - 1, p % c.page] = values.to(c.kv_type)
        for t in range(c.starts[r], c.starts[r + 1]):
            at = c.lens[r] - (c.starts[r + 1] - t)
            if p <= at and (c.window == 0 or p > at - c.window or p < c.sinks):
                bad[t, k::STEP] = True
    return bad


def _check(c, bad, only):
    got = c.out_d[:c.total].double().cpu().numpy()
    heads = c.kv * c.group
    finite = np.isfinite(got)
    wrong = finite == np.broadcast_to(bad[:, None], finite.shape)
    assert not wrong.any(), f"tokens {sorted(set(np.nonzero(wrong)[0].tolist()))[:20]} of {wrong.any((1, 2)).sum()}"
    lse = c.lse_d[:c.total].double().cpu().numpy()
    h, n = HALF[c.q_type], max([1] + c.lens)
    with np.errstate(invalid="ignore"):
        want = c.exact(only=only)
    assert len(want) == len(only) * heads
    for (t, head), (o, l, spread, size) in want.items():              # the bounds of test_gpu_attention.py
        dx = (c.dim + 4) * U * size
        sums = 2.0 ** -22 + (n + 64) * U
        fine = ~bad[t]
        bound = h * np.abs(o) + spread * (1 + h) * (h + 2 * dx + sums) + TINY[c.q_type]
        assert (np.abs(got[t, head][fine] - o[fine]) <= bound[fine]).all(), (t, head)
        if l == -np.inf:
            assert lse[t, head] == -np.inf
        else:
            assert abs(lse[t, head] - l) <= dx + sums + 2.0 ** -22 * abs(l), (t, head)


KINDS = [dict(group=4), dict(group=1), dict(group=3), dict(group=8, kv=1), dict(group=2, dim=64, kv=3),
         dict(group=4, dim=256, kv=1), dict(group=1, dim=96, page=24, major="head"), dict(group=4, q_type=FP, kv_type=FP),
         dict(group=1, kv_type=F8), dict(group=5, q_type=FP, kv_type=F8, dim=64), dict(group=2, dim=25),
         dict(group=4, window=70), dict(group=1, window=40, sinks=12, q_type=FP, kv_type=FP), dict(group=2, window=130, sinks=5, kv_type=F8)]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
def test_prompt_values(tk, kind, junk):  # noqa: F811
    """Whole prompts and chunks that start inside key tiles."""
    say(f"[attention] values of {junk}, prompt {KINDS[kind]}")
    lens, news = [90, 256, 1, 201], [75, 256, 1, 130]
    c = Case(300 + kind, lens, news, **KINDS[kind])
    bad = _spoil(c, [(0, 41, 0), (0, 3, 1), (1, 10, 0), (1, 127, 2), (1, 128, 3), (1, 255, 4), (3, 64, 1), (3, 100, 0)], junk)
    assert bad.any() and not bad.all()
    c.device(tk)
    c.call(tk)
    _check(c, bad, set(range(0, c.total, 5)) | {40, 41, 42, 85})


@pytest.mark.parametrize("lens,news,kw", [
    ([5000], [512], dict(group=8, kv=1, q_type=FP, kv_type=FP)),      # few row tiles behind a long cache: cut along the keys
    ([3001, 77], [64, 50], dict(group=4, kv=8)), ([5000, 4000], [3, 70], dict(group=4, kv=1, kv_type=F8)),
    ([6000], [100], dict(group=1, kv=2, dim=64, window=3000, sinks=7)), ([2500], [33], dict(group=4, kv=1, dim=256)),
    ([2230, 65], [2230, 65], dict(group=8, kv=8)),                    # row tiles that fill the GPU by themselves
    ([2230, 65], [2230, 65], dict(group=8, kv=8, kv_type=F8)), ([1300, 1000], [1300, 900], dict(group=5, kv=16, window=1030, sinks=9))])
def test_long_prompt_values(tk, lens, news, kw):  # noqa: F811
    say(f"[attention] values of NaN, {news} of {lens} {kw}")
    c = Case(17, lens, news, **kw)
    n, m = lens[0], lens[0] - news[0]
    spoils = [(0, m + 5 * news[0] // 6, 0), (0, m + news[0] // 2, 1), (0, max(0, m - 40), 2), (0, m + news[0] // 4, 3),
              (len(lens) - 1, lens[-1] - news[-1] // 3 - 1, 4)]
    if kw.get("group") == 8 and news[0] == 512:
        spoils.append((0, 4600, 0))
    bad = _spoil(c, spoils, float("nan"))
    assert bad.any() and not bad.all()
    c.device(tk)
    c.call(tk)
    near = {c.starts[r] + p - (lens[r] - news[r]) + d for r, p, _ in spoils for d in (-1, 0, 1, 20)}
    _check(c, bad, {int(t) for t in near if 0 <= t < c.total} | {0, c.total - 1})


@pytest.mark.parametrize("kw", [dict(), dict(kv_type=F8), dict(q_type=FP, kv_type=FP, dim=64), dict(dim=25), dict(dim=256, kv=1),
                                dict(window=30, sinks=2)])
def test_decode_values(tk, kw):  # noqa: F811
    """Requests that are cut among them."""
    say(f"[attention] values of NaN, decode {kw}")
    c = Case(19, [5000, 40, 700, 1], **kw)
    bad = _spoil(c, [(0, 4990, 0), (0, 100, 1), (2, 690, 2), (2, 1, 3), (3, 0, 4)], float("nan"))
    c.device(tk)
    c.call(tk)
    _check(c, bad, {0, 1, 2, 3})
