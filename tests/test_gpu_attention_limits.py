"""Attention calls at the ends of what their options allow."""
import numpy as np
import pytest
import torch

from gpu_util import say
from test_gpu_attention import BF, F8, FP, Case, tk  # noqa: F401

pytestmark = pytest.mark.gpu
MOST = 2**31 - 1


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("kw", [dict(group=4), dict(group=1), dict(group=1, dim=64, q_type=FP, kv_type=FP), dict(dim=25, kv=1),
                                dict(group=2, kv_type=F8, dim=256, kv=1), dict(planes=1, kv=1, group=4, dim=576, value=512)])
@pytest.mark.parametrize("window,sinks", [(MOST, 0), (MOST, MOST), (MOST - 40, 3), (1 << 30, 0), (5, MOST)])
def test_windows_past_every_cache(tk, decode, kw, window, sinks):  # noqa: F811
    """A window wider than any cache hides nothing, also from the first tokens that the request really holds where the call
    names more new tokens than that; first tokens without number hide nothing either."""
    say(f"[attention] window {window}, first tokens {sinks}, {kw} decode={decode}")
    c = Case(71, [9, 100, 20, 0, 300], None if decode else [40, 130, 90, 3, 20], window=window, sinks=sinks, **kw).device(tk)
    c.call(tk)
    c.window = 0                                                       # the oracle's answer without one
    c.check()


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("kw", [dict(), dict(q_type=FP, kv_type=FP, dim=64), dict(kv_type=F8, window=60, sinks=2), dict(dim=25, kv=1),
                                dict(planes=1, kv=1, group=4, dim=576, value=512), dict(planes=1, kv=1, group=40, dim=576, value=512)])
def test_scale_below_normal_numbers(tk, decode, kw):  # noqa: F811
    """A scale that is a subnormal float makes all scores alike and no masked key visible."""
    say(f"[attention] scale 2^-140, {kw} decode={decode}")
    c = Case(73, [300, 1, 77, 0], None if decode else [90, 1, 77, 2], **kw)
    c.scale = 2.0 ** -140 / 0.75 if c.kv_type == F8 else 2.0 ** -140     # the e4m3 keys' factor is 0.75
    c.device(tk)
    c.call(tk)
    c.check()


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("v_scale", [0.0, -2.0, 1024.0])
def test_value_scales(tk, decode, v_scale):  # noqa: F811
    """Any finite factor of the values: none, negative, large; lse does not know of it."""
    say(f"[attention] v_scale {v_scale} decode={decode}")
    for kw in (dict(), dict(dim=25, kv=1), dict(planes=1, kv=1, group=4, dim=576, value=512)):
        c = Case(79, [2000, 60, 0], None if decode else [50, 60, 0], **kw)
        c.v_scale = v_scale
        c.device(tk)
        c.call(tk)
        c.check()


@pytest.mark.parametrize("reqs,kw", [(512, dict(group=2, kv=1, dim=64)), (513, dict(group=2, kv=1, dim=64)), (64, dict(group=1, kv=8)),
                                     (65, dict(group=1, kv=8)), (256, dict(planes=1, kv=1, group=3, dim=576, value=512)),
                                     (257, dict(planes=1, kv=1, group=3, dim=576, value=512))])
def test_decode_as_many_requests_as_shares(tk, reqs, kw):  # noqa: F811
    """Requests as many as the shares that the batch is cut into, and one more; most of them short, some cut."""
    say(f"[attention] {reqs} requests {kw}")
    rng = np.random.default_rng(reqs)
    lens = rng.integers(0, 40, reqs)
    lens[[0, reqs // 3, reqs - 2]] = [3000, 1500, 2900]
    c = Case(reqs, lens.tolist(), **kw).device(tk)
    c.call(tk)
    c.check(c.exact(only={0, 1, reqs // 3, reqs // 3 + 1, reqs - 3, reqs - 2, reqs - 1} | set(rng.integers(0, reqs, 60).tolist())))


@pytest.mark.parametrize("kw", [dict(group=2, kv=1, dim=64), dict(group=8, kv=1), dict(group=4, kv=2, kv_type=F8),
                                dict(group=2, kv=1, dim=256, q_type=FP, kv_type=FP), dict(group=4, kv=2, window=1000, sinks=30)])
@pytest.mark.parametrize("reqs,most", [(700, 5), (9, 4), (40, 300)])
def test_prompt_few_tokens_of_many_requests(tk, kw, reqs, most):  # noqa: F811
    """Drafts of a few tokens and chunks behind caches of very uneven length: row tiles cut along the keys, whole ones and
    requests without tokens side by side."""
    say(f"[attention] up to {most} tokens of {reqs} requests {kw}")
    rng = np.random.default_rng(reqs + most)
    lens = rng.integers(0, 60, reqs)
    some = [0, reqs // 2, reqs - 2]
    lens[some] = [3000, 1700, 2900]
    news = [int(rng.integers(0, min(int(n), most) + 1)) for n in lens]
    for r in some:
        news[r] = most
    c = Case(reqs, lens.tolist(), news, **kw).device(tk)
    c.call(tk)
    ends = {int(c.starts[r]) + d for r in some for d in (0, most // 2, most - 1)}
    c.check(c.exact(only=ends | set(rng.integers(0, c.total, 50).tolist())))


@pytest.mark.parametrize("kw", [dict(), dict(kv=1, group=8), dict(dim=25, kv=1), dict(dim=64, kv_type=F8)])
@pytest.mark.parametrize("starts", [[0, 100, 50, 120], [120, 0, 120, 0], [7, -3, 2**31 - 1, 5], [-2**31, 2**31 - 1, -2**31, 2**31 - 1]])
def test_starts_that_do_not_ascend(tk, kw, starts):  # noqa: F811
    """Nothing outside q's rows is written, and a good call afterwards is right: the workspace keeps nothing."""
    say(f"[attention] q_starts {starts} {kw}")
    c = Case(83, [900, 30, 70], [60, 20, 40], **kw).device(tk)
    good = c.starts_d.clone()
    c.starts_d.copy_(torch.tensor(starts, dtype=torch.int64).to(torch.int32).cuda())
    c.call(tk)
    torch.cuda.synchronize()
    assert (c.out_full[c.total:] == 77).all() and (c.lse_d[c.total:] == 77).all()
    c.starts_d.copy_(good)
    c.call(tk)
    c.check()
