"""Refusals of the attention and page calls, before any launch (no GPU needed)."""
import ctypes

import pytest

from test_abi_cpu import _expect, _pool, tk  # noqa: F401


def _view(tk, pool, layout=None, **kw):  # noqa: F811
    g = dict(layout=tk.TOPKV_LAYOUT_POOL if layout is None else layout, layer=0, head_begin=0, bt_stride=4,
             block_tables=0x20000, pool=pool, data=0, bytes=0, shards=0, reserved=0)
    g.update(kw)
    return tk.topkv_view_t(*[g[k] for k, _ in tk.topkv_view_t._fields_])


def _options(tk, **kw):  # noqa: F811
    g = dict(dtype=tk.TOPKV_BF16, kv_dtype=tk.TOPKV_BF16, num_heads=16, kv_heads=8, value_dim=128, window=0, sinks=0,
             reserved=0, scale=0.1, k_scale=1.0, v_scale=1.0, reserved2=0.0, q_stride=16 * 128, out_stride=16 * 128)
    g.update(kw)
    return tk.topkv_attention_t(*[g[k] for k, _ in tk.topkv_attention_t._fields_])


def _decode(tk, view, opt, reqs=2, lens=0x30000, q=0x40000, out=0x50000, lse=0, ws=0x1000000, wsb=1 << 40):  # noqa: F811
    tk.topkv_attention_decode(view, opt, reqs, lens, q, out, ws, lse=lse, workspace_bytes=wsb, stream=0)


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(dtype=3), dict(dtype=-1), dict(kv_dtype=1), dict(kv_dtype=2), dict(kv_dtype=7), dict(num_heads=0),
    dict(num_heads=12), dict(num_heads=-16), dict(kv_heads=0), dict(kv_heads=9), dict(kv_heads=-8), dict(value_dim=64),
    dict(value_dim=0), dict(value_dim=129), dict(window=-1), dict(sinks=-1), dict(reserved=1), dict(scale=0.0),
    dict(scale=-0.1), dict(scale=INF), dict(scale=NAN), dict(k_scale=0.0), dict(k_scale=-1.0), dict(k_scale=NAN),
    dict(v_scale=NAN), dict(v_scale=INF), dict(reserved2=1.0), dict(scale=1e30, k_scale=1e30),
    dict(scale=1e-40, k_scale=1e-40), dict(q_stride=2047), dict(out_stride=0)])
def test_attention_options_refused(tk, kw):  # noqa: F811
    view, opt = _view(tk, _pool(tk)), _options(tk, **kw)
    _expect(tk, tk.TOPKV_ERR_INVALID_ARG, lambda stream: _decode(tk, view, opt))
    with pytest.raises(tk.TopkvError):
        tk.topkv_attention_workspace_bytes(view, opt, 2, 2)


def test_attention_views_refused(tk):  # noqa: F811
    INV, UNS, opt = tk.TOPKV_ERR_INVALID_ARG, tk.TOPKV_ERR_UNSUPPORTED, _options(tk)
    good = _pool(tk)
    for view in (_view(tk, good, layout=tk.TOPKV_LAYOUT_PACKED), _view(tk, good, layout=3), _view(tk, good, layer=2),
                 _view(tk, good, layer=-1), _view(tk, good, head_begin=1), _view(tk, good, head_begin=-1),
                 _view(tk, good, bt_stride=0), _view(tk, good, block_tables=0), _view(tk, good, reserved=1),
                 _view(tk, _pool(tk, base=0)), _view(tk, _pool(tk, planes=3)), _view(tk, _pool(tk, elem_bytes=1)),
                 _view(tk, _pool(tk, elem_bytes=4)), _view(tk, _pool(tk, page_size=0))):
        _expect(tk, INV, lambda stream: _decode(tk, view, opt))
    _expect(tk, UNS, lambda stream: _decode(tk, _view(tk, good, bt_stride=1 << 28), opt))
    _expect(tk, UNS, lambda stream: _decode(tk, _view(tk, good), opt, reqs=tk.TOPKV_MAX_BATCH_REQS + 1))
    wide = _options(tk, num_heads=8, kv_heads=8, value_dim=1032, q_stride=8 * 1032, out_stride=8 * 1032)
    _expect(tk, UNS, lambda stream: _decode(tk, _view(tk, _pool(tk, head_dim=1032)), wide))
    _expect(tk, UNS, lambda stream: tk.topkv_attention_prompt(_view(tk, good), opt, 1, 0x1000, 0x2000, 1 << 28, 0x4000,
                                                              0x5000, 0x10000, workspace_bytes=1 << 40, stream=0))


def test_attention_pointers_refused(tk):  # noqa: F811
    INV, opt, view = tk.TOPKV_ERR_INVALID_ARG, _options(tk), _view(tk, _pool(tk))
    for kw in (dict(lens=0), dict(q=0), dict(out=0), dict(q=0x40001), dict(out=0x50001), dict(lse=0x60002),
               dict(reqs=-1)):
        _expect(tk, INV, lambda stream: _decode(tk, view, opt, **kw))
    prompt = tk.topkv_attention_prompt
    for kw in (dict(q_starts=0), dict(total_q=-1), dict(seq_lens=0)):
        a = dict(num_reqs=1, seq_lens=0x1000, q_starts=0x2000, total_q=3, q=0x4000, out=0x50000, workspace=0x10000,
                 workspace_bytes=1 << 40)
        a.update(kw)
        _expect(tk, INV, prompt, view, opt, **a)
    lib = ctypes.CDLL(tk.LIBRARY)
    assert lib.topkv_attention_decode(None, None, 1, None, None, None, None, None, ctypes.c_int64(0), None) == INV
    lib.topkv_attention_workspace_bytes.restype = ctypes.c_int64
    assert lib.topkv_attention_workspace_bytes(None, None, 1, 1) == -1


def test_attention_nothing_to_do(tk):  # noqa: F811
    opt, view = _options(tk), _view(tk, _pool(tk))
    _decode(tk, view, opt, reqs=0, lens=0, q=0, out=0)
    tk.topkv_attention_prompt(view, opt, 0, 0, 0, 5, 0, 0, 0x10000, workspace_bytes=1 << 40, stream=0)
    tk.topkv_attention_prompt(view, opt, 3, 0, 0, 0, 0, 0, 0x10000, workspace_bytes=1 << 40, stream=0)


@pytest.mark.parametrize("planes,dim,value", [(2, 64, 64), (2, 128, 128), (2, 256, 256), (1, 576, 512), (1, 64, 48), (2, 25, 25)])
@pytest.mark.parametrize("window", [0, 100, 4000])
def test_attention_workspace_serves_smaller_calls(tk, planes, dim, value, window):  # noqa: F811
    """What suffices for many requests and tokens suffices for fewer."""
    pool = _pool(tk, planes=planes, head_dim=dim)
    for heads, kv in ((8, 1), (16, 8), (128, 1)):
        opt = _options(tk, num_heads=heads, kv_heads=kv, value_dim=value, window=window, q_stride=heads * dim,
                       out_stride=heads * value)
        for stride in (4, 3000, 15000):
            view, most = _view(tk, pool, bt_stride=stride), -1
            for n in (0, 1, 7, 300, 4096):
                for total in (n, 3 * n + 100, 200000):
                    most = max(most, tk.topkv_attention_workspace_bytes(view, opt, n, total))
                    assert tk.topkv_attention_workspace_bytes(view, opt, 4096, 1 << 20) >= most


def _owner(tk, **kw):  # noqa: F811
    g = dict(ref_counts=0x1000, block_tables=0x2000, seq_lens=0x3000, num_pages=100, page_size=16, num_rows=4, bt_stride=8,
             reserved=0)
    g.update(kw)
    return tk.topkv_page_owner_t(*[g[k] for k, _ in tk.topkv_page_owner_t._fields_])


@pytest.mark.parametrize("kw", [dict(ref_counts=0), dict(block_tables=0), dict(seq_lens=0), dict(num_pages=0),
                                dict(num_pages=1 << 31), dict(num_pages=-4), dict(page_size=0), dict(num_rows=0),
                                dict(bt_stride=0), dict(reserved=2), dict(bt_stride=1 << 28)])
def test_owners_refused(tk, kw):  # noqa: F811
    INV, o = tk.TOPKV_ERR_INVALID_ARG, _owner(tk, **kw)
    big = dict(workspace_bytes=1 << 40, max_pairs=1 << 30)
    _expect(tk, INV, tk.topkv_pages_count, o, 0x9000)
    _expect(tk, INV, tk.topkv_pages_free, o, 1, 0x4000, 0x9000)
    _expect(tk, INV, tk.topkv_pages_fork, o, 1, 0x4000, 0x5000, 0x6000, 0x10000, 0x9000, **big)
    _expect(tk, INV, tk.topkv_pages_grow, o, 1, 0x4000, 0x5000, 0x6000, 0x10000, 0x9000, **big)
    _expect(tk, INV, tk.topkv_pages_compact, o, 0x6000, 0x10000, 0x9000, **big)
    with pytest.raises(tk.TopkvError):
        tk.topkv_pages_workspace_bytes(o)


def test_page_arguments_refused(tk):  # noqa: F811
    INV, o = tk.TOPKV_ERR_INVALID_ARG, _owner(tk)
    need = tk.topkv_pages_workspace_bytes(o)
    assert need > 0 and need % 4 == 0
    _expect(tk, INV, tk.topkv_pages_count, o, 0)
    for num, rows, result in ((-1, 0x4000, 0x9000), (1, 0, 0x9000), (1, 0x4000, 0),
                              (tk.TOPKV_MAX_BATCH_REQS + 1, 0x4000, 0x9000)):
        _expect(tk, INV, tk.topkv_pages_free, o, num, rows, result)
    for call in (tk.topkv_pages_fork, tk.topkv_pages_grow):
        good = dict(num=2, a=0x4000, b=0x5000, pairs=0x6000, work=0x10000, result=0x9000, most=2, room=need)
        for kw in (dict(num=-1), dict(num=5), dict(a=0), dict(b=0), dict(pairs=0), dict(work=0), dict(result=0), dict(most=1),
                   dict(room=need - 1), dict(work=0x10008)):
            g = {**good, **kw}
            _expect(tk, INV, call, o, g["num"], g["a"], g["b"], g["pairs"], g["work"], g["result"], max_pairs=g["most"],
                    workspace_bytes=g["room"])
    for kw in (dict(pairs=0), dict(most=49), dict(work=0), dict(room=need - 1), dict(result=0), dict(work=0x10004)):
        g = {**dict(pairs=0x6000, work=0x10000, result=0x9000, most=50, room=need), **kw}
        _expect(tk, INV, tk.topkv_pages_compact, o, g["pairs"], g["work"], g["result"], max_pairs=g["most"],
                workspace_bytes=g["room"])


def test_copy_pages_refused(tk):  # noqa: F811
    INV, UNS, good = tk.TOPKV_ERR_INVALID_ARG, tk.TOPKV_ERR_UNSUPPORTED, _pool(tk)
    copy = tk.topkv_copy_pages
    for other in (dict(planes=1), dict(page_size=32), dict(num_heads=4), dict(head_dim=64), dict(elem_bytes=4), dict(base=0),
                  dict(page_size=0)):
        _expect(tk, INV, copy, good, _pool(tk, **other), 0, 2, 0x6000, max_pairs=3)
        _expect(tk, INV, copy, _pool(tk, **other), good, 0, 2, 0x6000, max_pairs=3)
    for first, layers, pairs, most in ((-1, 1, 0x6000, 3), (0, 3, 0x6000, 3), (2, 1, 0x6000, 3), (0, -1, 0x6000, 3),
                                       (0, 2, 0, 3), (0, 2, 0x6000, -1)):
        _expect(tk, INV, copy, good, good, first, layers, pairs, max_pairs=most)
    _expect(tk, INV, copy, good, _pool(tk, num_layers=1), 1, 1, 0x6000, max_pairs=3)
    _expect(tk, UNS, copy, _pool(tk, num_pages=1 << 40, num_layers=1 << 20), good, 0, 1, 0x6000, max_pairs=3)
    copy(good, good, 0, 0, 0, max_pairs=3, stream=0)
    copy(good, good, 0, 2, 0, max_pairs=0, stream=0)


def _ints(*shape):
    import torch
    return torch.zeros(shape, dtype=torch.int32)


def test_short_tensors_refused(tk):  # noqa: F811
    """Index tensors that are shorter than the call reads or writes never reach the library."""
    view, opt, o = _view(tk, _pool(tk)), _options(tk), _owner(tk)
    need = tk.topkv_pages_workspace_bytes(o)
    room = dict(workspace_bytes=1 << 40, stream=0)
    page = dict(max_pairs=9, workspace_bytes=need, stream=0)
    calls = [
        lambda: tk.topkv_attention_decode(view, opt, 3, _ints(2), 0x4000, 0x5000, 0x10000, **room),
        lambda: tk.topkv_attention_prompt(view, opt, 3, _ints(2), 0x3000, 5, 0x4000, 0x5000, 0x10000, **room),
        lambda: tk.topkv_attention_prompt(view, opt, 3, 0x3000, _ints(3), 5, 0x4000, 0x5000, 0x10000, **room),
        lambda: tk.page_owner(_ints(10), 0x2000, 0x3000, page_size=16, num_pages=11, num_rows=2, bt_stride=4),
        lambda: tk.page_owner(0x1000, _ints(2, 4), 0x3000, page_size=16, num_pages=11, num_rows=2, bt_stride=5),
        lambda: tk.page_owner(0x1000, 0x2000, _ints(1), page_size=16, num_pages=11, num_rows=2, bt_stride=4),
        lambda: tk.topkv_pages_count(o, _ints(3), stream=0),
        lambda: tk.topkv_pages_free(o, 3, _ints(2), 0x9000, stream=0),
        lambda: tk.topkv_pages_free(o, 3, 0x4000, 0x9000, _ints(2), stream=0),
        lambda: tk.topkv_pages_free(o, 3, 0x4000, _ints(3), stream=0),
        lambda: tk.topkv_pages_fork(o, 3, _ints(2), 0x5000, 0x6000, 0x10000, 0x9000, **page),
        lambda: tk.topkv_pages_fork(o, 3, 0x4000, _ints(2), 0x6000, 0x10000, 0x9000, **page),
        lambda: tk.topkv_pages_fork(o, 3, 0x4000, 0x5000, _ints(8, 2), 0x10000, 0x9000, **page),
        lambda: tk.topkv_pages_fork(o, 3, 0x4000, 0x5000, 0x6000, 0x10000, _ints(1), **page),
        lambda: tk.topkv_pages_grow(o, 3, _ints(2), 0x5000, 0x6000, 0x10000, 0x9000, **page),
        lambda: tk.topkv_pages_grow(o, 3, 0x4000, _ints(1), 0x6000, 0x10000, 0x9000, **page),
        lambda: tk.topkv_pages_grow(o, 3, 0x4000, 0x5000, 0x6000, 0x10000, _ints(0), **page),
        lambda: tk.topkv_pages_compact(o, _ints(8, 2), 0x10000, 0x9000, **page),
        lambda: tk.topkv_pages_compact(o, 0x6000, 0x10000, _ints(3), max_pairs=50, workspace_bytes=need, stream=0),
        lambda: tk.topkv_copy_pages(_pool(tk), _pool(tk), 0, 1, _ints(2, 2), max_pairs=3, stream=0),
        lambda: tk.topkv_copy_pages(_pool(tk), _pool(tk), 0, 1, 0x6000, max_pairs=3, count=_ints(0), stream=0)]
    for call in calls:
        with pytest.raises(ValueError, match="at least"):
            call()
