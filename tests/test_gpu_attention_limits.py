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
