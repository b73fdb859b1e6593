"""Attention over a paged cache through the C ABI vs the 64-bit oracle.

Bounds, from the arithmetic (h = half a step of a type relative to the value, HALF; u = 2^-24):
  score   x = scale * q.k in 32 bits over D products: |dx| <= (D + 4) u * size, size = max_j scale sum |q_d k_jd|
  weight  p = exp(x): relative 2 |dx| at most with its normaliser, 2^-22 for the power of two itself, and one rounding to
          the inputs' type before the product with the values (h)
  sums    n terms in 32 bits: n u relative to sum p |v| (spread)
  result  one rounding to the output type: h |out|; below the type's smallest normal number half its step there
so |out - exact| <= h |exact| + spread (1 + h) (h + 2 |dx| + 2^-22 + (n + 64) u) + tiny.
  lse     |dx| + 2^-22 + (n + 64) u, and 2^-22 of its own size for the logarithm's 32 bits."""
import numpy as np
import pytest
import torch

from gpu_util import say, to_dev
from oracle.attention import attend

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # torch.finfo(t).eps / 2
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U = 2.0 ** -24
BF, FP, F8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def tk():
    from paper_2607_28633_amd import topkv
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return topkv


class Case:
    """A pool whose unused places hold NaN (e4m3: its NaN) or infinities, tables, queries."""

    def __init__(self, seed, lens, news=None, planes=2, kv=2, group=4, dim=128, value=None, page=16, major="slot", q_type=BF,
                 kv_type=BF, window=0, sinks=0, extra_heads=0, layers=1, layer=0, junk=float("nan"), q_pad=0, spread=1.0,
                 wide=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.decode = list(lens), news is None
        self.news = [1] * len(lens) if news is None else list(news)
        self.planes, self.kv, self.group, self.dim = planes, kv, group, dim
        self.value = dim if value is None else value
        self.page, self.major, self.window, self.sinks, self.layer, self.layers = page, major, window, sinks, layer, layers
        self.q_type, self.kv_type, self.head_begin = q_type, kv_type, extra_heads
        need = [-(-max(0, n) // page) for n in lens]
        stride = max([1] + need) + 1 + wide
        pages = sum(need) + 3
        perm = torch.randperm(pages, generator=g).tolist()
        self.tables = np.full((len(lens), stride), -1, dtype=np.int32)
        heads = kv + extra_heads
        pool = torch.full((pages, planes, page, heads, dim), junk)     # slot-major, floats
        at = 0
        for r, n in enumerate(lens):
            for j in range(need[r]):
                p = perm[at]
                at += 1
                self.tables[r, j] = p
                k = min(page, n - j * page)
                pool[p, :, :k] = torch.randn((planes, k, heads, dim), generator=g)
        self.pool = pool.to(kv_type)
        self.total = sum(self.news)
        self.starts = np.concatenate([[0], np.cumsum(self.news)]).astype(np.int32)
        self.q = (torch.randn((self.total, kv * group, dim + q_pad), generator=g) * spread).to(q_type)[..., :dim]
        self.q_pad = q_pad
        self.scale = 1.0 / np.sqrt(dim)
        self.k_scale, self.v_scale = (0.75, 1.25) if kv_type == F8 else (1.0, 1.0)

    def exact(self, only=None):
        pool = self.pool.to(torch.float64).numpy()
        pool = pool * self.k_scale
        got = attend(pool, self.tables, [max(0, min(n, self.tables.shape[1] * self.page)) for n in self.lens], self.starts,
                     self.q.to(torch.float64).numpy(), self.kv, self.scale, self.value, self.window, self.sinks,
                     self.head_begin, only)
        return {k: (o * (self.v_scale / self.k_scale), l, s * abs(self.v_scale / self.k_scale), b)
                for k, (o, l, s, b) in got.items()}

    def device(self, tk):
        pool = self.pool
        if self.major == "head":
            pool = pool.transpose(2, 3).contiguous()
        bytes_ = pool.contiguous().view(torch.uint8)
        full = torch.full((self.layers,) + tuple(bytes_.shape), 0x7F, dtype=torch.uint8)   # other layers: NaN in every type
        full[self.layer] = bytes_
        self.pool_d = full.cuda().view(self.kv_type)
        self.tables_d, self.lens_d = to_dev(self.tables), to_dev(np.array(self.lens, dtype=np.int32))
        self.starts_d = to_dev(self.starts)
        wide = torch.zeros((self.total, self.q.shape[1] * self.dim + self.q_pad * 8), dtype=self.q_type)
        wide[:, :self.q.shape[1] * self.dim] = self.q.reshape(self.total, -1)
        self.q_d = wide.cuda()[:, :self.q.shape[1] * self.dim].view(self.total, self.q.shape[1], self.dim) \
            if self.q_pad == 0 else wide.cuda()[:, :self.q.shape[1] * self.dim].unflatten(1, (self.q.shape[1], self.dim))
        rows = self.total + 2
        out = torch.full((rows, self.q.shape[1] * self.value + self.q_pad * 8), 77.0, dtype=self.q_type, device="cuda")
        self.out_full = out
        self.out_d = out[:, :self.q.shape[1] * self.value].unflatten(1, (self.q.shape[1], self.value))
        self.lse_d = torch.full((rows, self.q.shape[1]), 77.0, device="cuda")
        self.cache = tk.pool_view(self.pool_d, self.layer, self.tables_d, self.tables.shape[1], self.head_begin,
                                  self.major == "head")
        self.options = tk.attention_options(self.q_d, self.out_d[:self.total], kv_heads=self.kv, scale=self.scale,
                                            kv_dtype=self.kv_type, window=self.window, sinks=self.sinks, k_scale=self.k_scale,
                                            v_scale=self.v_scale)
        room = tk.topkv_attention_workspace_bytes(self.cache, self.options, len(self.lens), self.total)
        self.work = torch.randint(0, 256, (room + 256,), dtype=torch.uint8, device="cuda")[:room]
        return self

    def call(self, tk, lse=True):
        kw = dict(lse=self.lse_d if lse else None, workspace=self.work)
        if self.decode:
            tk.topkv_attention_decode(self.cache, self.options, len(self.lens), self.lens_d, self.q_d, self.out_d, **kw)
        else:
            tk.topkv_attention_prompt(self.cache, self.options, len(self.lens), self.lens_d, self.starts_d, self.total,
                                      self.q_d, self.out_d, **kw)

    def check(self, want=None, lse=True):
        torch.cuda.synchronize()
        want = self.exact() if want is None else want
        got, got_lse = self.out_d.double().cpu().numpy(), self.lse_d.double().cpu().numpy()
        h = HALF[self.q_type]
        for (t, head), (o, l, spread, size) in want.items():
            n = max([1] + self.lens)
            dx = (self.dim + 4) * U * size
            rel = h + 2 * dx + 2.0 ** -22 + (n + 64) * U
            bound = h * np.abs(o) + spread * (1 + h) * rel + TINY[self.q_type]
            off = np.abs(got[t, head] - o)
            assert np.isfinite(got[t, head]).all(), f"token {t} head {head}: {got[t, head]}"
            assert (off <= bound).all(), f"token {t} head {head}: off {off.max()} of {bound[off.argmax()]}"
            if not lse:
                continue
            if l == -np.inf:
                assert got_lse[t, head] == -np.inf and (got[t, head] == 0).all()
            else:
                assert abs(got_lse[t, head] - l) <= dx + 2.0 ** -22 + (n + 64) * U + 2.0 ** -22 * abs(l), \
                    f"lse of token {t} head {head}: {got_lse[t, head]} against {l}"
        assert (self.out_full[self.total:] == 77).all() and (self.lse_d[self.total:] == 77).all()
        if self.q_pad:
            assert (self.out_full[:, self.q.shape[1] * self.value:] == 77).all()
        if not lse:
            assert (self.lse_d == 77).all()


SHAPES = [
    dict(),
    dict(q_type=FP, kv_type=FP),
    dict(kv_type=F8),
    dict(q_type=FP, kv_type=F8, dim=64),
    dict(dim=64, kv=3, group=5, major="head"),
    dict(dim=256, kv=1, group=16, page=64),
    dict(dim=96, kv=2, group=1, page=24),
    dict(dim=96, kv=2, group=3, kv_type=F8, page=1),
    dict(dim=80, group=7, q_type=FP, kv_type=FP, page=5, major="head"),
    dict(planes=1, kv=1, group=16, dim=576, value=512, page=64),
    dict(planes=1, kv=1, group=40, dim=576, value=512, page=16, q_type=FP, kv_type=FP),
    dict(planes=1, kv=2, group=3, dim=64, value=40, page=16),
    dict(planes=1, kv=1, group=9, dim=576, value=512, kv_type=F8),
    dict(dim=25, kv=7, group=2, page=9),
    dict(dim=200, kv=1, group=4, kv_type=F8),
    dict(dim=8, kv=1, group=1),
    dict(dim=1, kv=1, group=3, page=3),
    dict(dim=320, kv=1, group=2, q_type=FP, kv_type=FP),
    dict(dim=128, kv=1, group=33),
    dict(dim=128, kv=2, group=4, extra_heads=1, layers=3, layer=1),
    dict(dim=128, kv=2, group=4, q_pad=8),
    dict(dim=128, kv=2, group=4, q_pad=1),
]
MASKS = [dict(), dict(window=1), dict(window=128, sinks=4), dict(window=37), dict(window=100, sinks=300)]
LENS = [0, 1, 2, 15, 16, 17, 63, 130, 257, 700]


# every shape without a mask and with one, some shapes with all of them
BOTH = [(i, j) for i in range(len(SHAPES)) for j in range(len(MASKS)) if j == 0 or i % 4 == j % 4 or i in (0, 2, 9)]


@pytest.mark.parametrize("shape,mask", BOTH)
def test_decode(tk, shape, mask):
    say(f"[attention] decode {SHAPES[shape]} {MASKS[mask]}")
    c = Case(100 * shape + mask, LENS, **SHAPES[shape], **MASKS[mask]).device(tk)
    c.call(tk)
    c.check()


@pytest.mark.parametrize("shape,mask", BOTH)
def test_prompt(tk, shape, mask):
    """Whole prompts, chunks behind a cache, single tokens, none at all, more new tokens than the request holds."""
    say(f"[attention] prompt {SHAPES[shape]} {MASKS[mask]}")
    c = Case(100 * shape + mask, [33, 150, 70, 9, 0, 260, 40, 1], [33, 21, 1, 0, 2, 67, 45, 1], **SHAPES[shape],
             **MASKS[mask]).device(tk)
    c.call(tk)
    c.check()


@pytest.mark.parametrize("kw", [dict(), dict(dim=96, q_type=FP, kv_type=FP), dict(kv_type=F8), dict(window=1500, sinks=5),
                                dict(dim=120, page=24, major="head"), dict(dim=64), dict(dim=256, kv=4), dict(group=3, kv=16)])
def test_prompt_large(tk, kw):
    """Prompts that fill the GPU by themselves, with absent pages and tokens of NaN; rows checked at random and around
    those and the prompts' ends."""
    say(f"[attention] large prompt {kw}")
    lens = [2230, 1, 700, 65]
    c = Case(37, lens, lens, **{**dict(kv=8, group=8), **kw})
    rng = np.random.default_rng(1)
    c.tables[0, 300 // c.page] = -1
    c.tables[2, 650 // c.page] = 2**31 - 1
    page = c.pool[int(c.tables[0, 1500 // c.page])].to(torch.float32)
    page[-1, 1500 % c.page] = float("nan")                            # the value of token 1500
    c.pool[int(c.tables[0, 1500 // c.page])] = page.to(c.kv_type)
    c.device(tk)
    c.call(tk)
    first = int(c.starts[2])
    only = {0, 1, 62, 63, 64, 299, 320, 1400, 1490, 1498, 1499, 2230, 2231, first + 699, first + 650, first + 700}
    only |= set(rng.integers(0, 1500, 8).tolist()) | set((first + rng.integers(0, 700, 8)).tolist())
    with np.errstate(invalid="ignore"):
        c.check(c.exact(only=only))
    assert not torch.isfinite(c.out_d[1500].float()).any() and not torch.isfinite(c.out_d[1700].float()).any()
    c.out_full.fill_(77), c.lse_d.fill_(77)
    before = c.out_full.clone()
    c.call(tk)
    first_run = c.out_full.clone()
    c.call(tk)
    assert torch.equal(torch.nan_to_num(first_run), torch.nan_to_num(c.out_full)) and not torch.equal(before, c.out_full)


@pytest.mark.parametrize("lens,kw", [([5000], {}), ([20011, 3, 900], dict(group=8, kv=1)), ([4097] * 3, dict(kv_type=F8)),
                                     ([9000, 100], dict(planes=1, kv=1, group=16, dim=576, value=512, page=64)),
                                     ([30000, 17, 12000], dict(dim=64, window=5000, sinks=70)), ([6000], dict(dim=256, kv=1)),
                                     ([3000, 2999], dict(planes=1, kv=1, group=128, dim=576, value=512, page=16))])
def test_decode_long(tk, lens, kw):
    """Lengths that are split over many workgroups and joined; peaked scores."""
    say(f"[attention] long {lens} {kw}")
    c = Case(7, lens, spread=3.0, **kw).device(tk)
    c.call(tk)
    c.check()


@pytest.mark.parametrize("reqs", [65, 700, 4096])
def test_decode_many_requests(tk, reqs):
    say(f"[attention] {reqs} requests")
    rng = np.random.default_rng(reqs)
    lens = rng.integers(0, 12, reqs)
    lens[[3, reqs // 2, reqs - 1]] = [400, 1200, 90]
    c = Case(reqs, lens.tolist(), kv=1, group=2, dim=64).device(tk)
    c.call(tk)
    c.check()


def test_prompt_many_requests(tk):
    say("[attention] prompt of 1500 requests")
    rng = np.random.default_rng(2)
    lens = rng.integers(0, 30, 1500)
    news = [int(rng.integers(0, n + 1)) for n in lens]
    c = Case(5, lens.tolist(), news, kv=1, group=2, dim=64).device(tk)
    c.call(tk)
    c.check()


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("kw", [dict(), dict(kv_type=F8), dict(dim=64, window=50, sinks=3), dict(dim=25, kv=1),
                                dict(planes=1, kv=1, group=16, dim=576, value=512)])
def test_hostile_tables_and_lengths(tk, decode, kw):
    """Entries that are no page count as absent tokens; lengths past the table are cut to it, negative ones are none."""
    say(f"[attention] hostile {kw}")
    c = Case(11, [200, 90, 64, 130, 77], None if decode else [60, 90, 2, 5, 1], **kw)
    c.tables[0, [0, 3, 7]] = [-1, 2**31 - 1, c.pool.shape[0]]
    c.tables[1, :] = -2**31
    c.tables[2, 3] = -1
    c.lens[4] = -5
    c.device(tk)
    c.call(tk)
    want = c.exact()
    c.check(want)
    # a length past the table: the table's last, invalid entry stands for absent tokens
    # (request 2 has only whole pages; request 3's last page is partial, so its length now covers stale NaN)
    for r in (2, 3):
        c.lens_d[r] = 2**31 - 1
        c.lens[r] = c.tables.shape[1] * c.page
    c.call(tk)
    want = c.exact()
    c.check({k: w for k, w in want.items() if np.isfinite(w[0]).all()})
    assert all(not torch.isfinite(c.out_d[k]).all() for k, w in want.items() if not np.isfinite(w[0]).all())


@pytest.mark.parametrize("kw", [dict(), dict(dim=64, kv=1, group=8), dict(dim=25, kv=1), dict(q_type=FP, kv_type=FP, dim=256),
                                dict(window=30, sinks=2), dict(kv_type=F8), dict(planes=1, kv=1, group=4, dim=576, value=512)])
@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
def test_prompt_tokens_to_come_do_not_reach_back(tk, kw, junk):
    """A token whose key and value hold NaN or infinities leaves every earlier token's result as it is."""
    say(f"[attention] junk ahead {kw} {junk}")
    c = Case(13, [90, 50], [75, 50], **kw)
    spoiled = {0: 41, 1: 17}                                          # request -> position
    for r, p in spoiled.items():
        page = c.pool[int(c.tables[r, p // c.page])].to(torch.float32)
        page[:, p % c.page, :, ::3] = junk
        c.pool[int(c.tables[r, p // c.page])] = page.to(c.kv_type)
    c.device(tk)
    c.call(tk)
    with np.errstate(invalid="ignore", over="ignore"):
        want = c.exact()
    clean = {}
    for (t, h), w in want.items():
        r = 0 if t < 75 else 1
        pos = c.lens[r] - (c.starts[r + 1] - t)
        seen = spoiled[r] <= pos and (not c.window or spoiled[r] > pos - c.window or spoiled[r] < c.sinks)
        if not seen:
            clean[t, h] = w
    assert clean and len(clean) < len(want)
    c.check(clean)
    # rows that do see it are NaN or infinite in the spoiled values, as the formula has it
    bad = [k for k in want if k not in clean]
    assert all(not torch.isfinite(c.out_d[t, h]).all() for t, h in bad)


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("kw", [dict(), dict(kv_type=F8), dict(q_type=FP, kv_type=FP, dim=64), dict(dim=25), dict(window=30, sinks=2),
                                dict(planes=1, kv=1, group=4, dim=576, value=512),
                                dict(planes=1, kv=1, group=40, dim=576, value=512)])
def test_queries_of_nan(tk, decode, kw):
    """A query with a NaN gives NaN, in requests that are cut too, and nothing to the rows beside it."""
    say(f"[attention] NaN queries {kw} decode={decode}")
    c = Case(53, [5000, 40, 1], None if decode else [3, 20, 1], **kw)
    spoiled = [(0, 1), (c.total - 1, 0)]
    for t, h in spoiled:
        c.q[t, h, c.dim // 2] = float("nan")
    c.device(tk)
    c.call(tk)
    c.check({k: w for k, w in c.exact().items() if k not in spoiled})
    for t, h in spoiled:
        assert torch.isnan(c.out_d[t, h]).all() and torch.isnan(c.lse_d[t, h])


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("kw", [dict(q_type=FP, kv_type=FP), dict(), dict(q_type=FP, kv_type=FP, dim=25),
                                dict(q_type=FP, kv_type=FP, planes=1, kv=1, group=4, dim=576, value=512),
                                dict(q_type=FP, kv_type=FP, planes=1, kv=1, group=64, dim=576, value=512),
                                dict(q_type=FP, kv_type=FP, dim=256), dict(q_type=FP, kv_type=F8, dim=64)])
def test_scores_past_24_bits(tk, decode, kw):
    """Scores so large that neighbouring 32-bit floats lie whole powers of two apart.  One key is far above the others: its
    weight is the only one, and the result its value.  The weight itself is rounded once (h), the result once more (h)."""
    say(f"[attention] large scores {kw} decode={decode}")
    lens = [300 + 7 * k for k in range(12)] + [2500, 2501]
    c = Case(59, lens, None if decode else [2] * len(lens), **kw)
    c.q[:] = 0
    c.q[..., 0] = 400.0                                            # with keys of 208 .. 416 and the scale: 2^15 .. 2^41
    c.scale, top = 1.0, 416.0
    keys = c.pool[:, 0]
    keys[..., 0] = torch.nan_to_num(keys[..., 0].float()).clamp(-10, 10).to(c.kv_type)
    won = []
    for r, n in enumerate(lens):
        j = (0, n // 2, n - 2)[r % 3]
        for i, at in enumerate((j // 3, j)):                       # one that is passed by, and the winner
            keys[int(c.tables[r, at // c.page]), at % c.page, :, 0] = (208.0, top)[i] if at < j or i else top
        won.append(j)
    c.device(tk)
    for power in range(-2, 25, 2):
        c.options.scale = 2.0 ** power
        c.out_full.fill_(77), c.lse_d.fill_(77)
        c.call(tk)
        torch.cuda.synchronize()
        got, lse = c.out_d.double().cpu(), c.lse_d.double().cpu()
        exact = 2.0 ** power * 400.0 * top * c.k_scale
        for t in range(c.total):
            r = t if decode else t // 2
            at, n = won[r], c.lens[r]
            row = c.pool[int(c.tables[r, at // c.page]), c.planes - 1, at % c.page].double() * c.v_scale
            for h in range(c.kv * c.group):
                v = row[h // c.group][:c.value]
                assert ((got[t, h] - v).abs() <= 2 * HALF[c.q_type] * v.abs() + TINY[c.q_type]).all(), (power, t, h)
                assert abs(lse[t, h] - exact) <= 8 * U * exact, (power, t, h)


@pytest.mark.parametrize("kw", [dict(), dict(dim=64), dict(window=200, sinks=3), dict(dim=256, kv=4)])
def test_large_prompt_scores_past_24_bits(tk, kw):
    """Whole prompts whose keys grow with their position, by steps of 100 e-folds and more: each token's result is its own
    value, rounded at most twice."""
    say(f"[attention] large prompt, large scores {kw}")
    lens = [1200, 1201]
    c = Case(61, lens, lens, q_type=FP, kv_type=FP, **{**dict(kv=8, group=8), **kw})
    c.q[:] = 0
    c.q[..., 0] = 400.0
    c.scale = 1.0
    values = []
    for r, n in enumerate(lens):
        at = np.arange(n)
        page, slot = torch.from_numpy(c.tables[r, at // c.page]).long(), torch.from_numpy(at % c.page)
        c.pool[page, 0, slot, :, 0] = torch.from_numpy(at).to(FP)[:, None].expand(n, c.kv)       # exact below 2048
        values.append(c.pool[page, 1, slot])
    v = torch.cat(values).double().repeat_interleave(c.group, 1)
    c.device(tk)
    for power in (-2, 10, 14, 18, 24):
        c.options.scale = 2.0 ** power
        c.out_full.fill_(77), c.lse_d.fill_(77)
        c.call(tk)
        torch.cuda.synchronize()
        got = c.out_d[:c.total].double().cpu()
        assert ((got - v).abs() <= 2 * HALF[FP] * v.abs() + TINY[FP]).all(), power


@pytest.mark.parametrize("decode", [True, False])
def test_many_small_weights(tk, decode):
    """One key far above 40000 others whose weights are each below half floats' normal numbers: together they count."""
    say("[attention] many small weights")
    n = 40001
    c = Case(41, [n], None if decode else [3], q_type=FP, kv_type=FP, kv=1, group=4, dim=64, page=64)
    c.q[:] = 0
    c.q[..., 0] = 8.0
    keys = c.pool[:, 0]
    keys[..., 0] = 0.0
    first = int(c.tables[0, 0])
    keys[first, 5, :, 0] = 10.375                                    # e^(8 * 10.375 / 8): each other weight is 3.1e-5
    c.pool[:, 1][..., ::2] = c.pool[:, 1][..., ::2].abs()
    c.device(tk)
    c.call(tk)
    c.check()


@pytest.mark.parametrize("which", ["cache", "q", "out", "all"])
@pytest.mark.parametrize("kw", [dict(), dict(kv_type=F8), dict(planes=1, kv=1, group=5, dim=576, value=512)])
def test_odd_addresses(tk, which, kw):
    """Pools, queries and outputs that start off 16-byte addresses."""
    say(f"[attention] {which} off alignment {kw}")
    for news in (None, [60, 5, 0]):
        c = Case(43, [300, 5, 90], news, **kw).device(tk)

        def moved(t):
            flat = torch.empty(t.untyped_storage().nbytes() + 64, dtype=torch.uint8, device="cuda")
            at = flat[2 if t.element_size() == 2 else 1:][:t.untyped_storage().nbytes()]
            at.copy_(torch.empty(0, dtype=torch.uint8, device="cuda").set_(t.untyped_storage()))
            c.keep = getattr(c, "keep", []) + [flat]
            return at.data_ptr()

        pool = c.pool_d
        if which in ("cache", "all"):
            c.cache.pool.base = moved(c.pool_d)
        q = moved(c.q_d) if which in ("q", "all") else c.q_d
        out, kept = c.out_d, c.out_full
        if which in ("out", "all"):
            flat = torch.full((kept.numel() + 8,), 77.0, dtype=kept.dtype, device="cuda")
            c.out_full = flat[1:1 + kept.numel()].view(kept.shape)
            c.out_d = c.out_full.unflatten(1, out.shape[1:])
        c.q_d = q
        if news is None:
            tk.topkv_attention_decode(c.cache, c.options, 3, c.lens_d, q, c.out_d.data_ptr(), c.work, lse=c.lse_d)
        else:
            tk.topkv_attention_prompt(c.cache, c.options, 3, c.lens_d, c.starts_d, c.total, q, c.out_d.data_ptr(), c.work,
                                      lse=c.lse_d)
        c.check()
        assert pool is c.pool_d


def test_tensors_are_looked_over(tk):
    """The binding refuses tensors that are not what the options describe."""
    c = Case(47, [30, 40]).device(tk)
    n, h, d = 2, 8, 128
    good = dict(q=c.q_d, out=c.out_d, lse=c.lse_d)
    for bad in (dict(q=c.q_d[:1]), dict(q=c.q_d[:, :4]), dict(q=c.q_d.half()), dict(q=c.q_d.cpu()),
                dict(out=torch.empty((n, h, 64), dtype=BF, device="cuda")), dict(q=torch.empty((n, 2 * h, d), dtype=BF, device="cuda")[:, ::2]),
                dict(q=torch.empty((n, 3 * h, d), dtype=BF, device="cuda")[:, :h]), dict(q=c.q_d[:1].expand(n, h, d)),
                dict(lse=torch.empty((n, h), dtype=torch.float64, device="cuda")), dict(lse=c.lse_d[:1]),
                dict(out=c.out_d.transpose(1, 2).contiguous().transpose(1, 2))):
        a = {**good, **bad}
        with pytest.raises(ValueError):
            tk.topkv_attention_decode(c.cache, c.options, n, c.lens_d, a["q"], a["out"], c.work, lse=a["lse"])
    with pytest.raises(ValueError):
        tk.attention_options(c.q_d, c.out_d.float(), kv_heads=2, scale=1.0)
    with pytest.raises(ValueError):
        tk.attention_options(c.q_d, c.out_d[:2], kv_heads=2, scale=1.0, kv_dtype=torch.int8)


def test_lse_is_optional(tk):
    for news in (None, [30, 5]):
        c = Case(3, [300, 5], news).device(tk)
        c.call(tk, lse=False)
        c.check(lse=False)


def test_rows_outside_requests_stay(tk):
    """q_starts that leave rows in front, between and behind: those keep their values."""
    say("[attention] rows of nobody")
    c = Case(17, [40, 60], [10, 30]).device(tk)
    q = torch.zeros((60,) + tuple(c.q_d.shape[1:]), dtype=BF, device="cuda")
    out = torch.full_like(q, 55)
    lse = torch.full((60, 8), 55.0, device="cuda")
    q[4:14], q[20:50] = c.q_d[:10], c.q_d[10:]
    opt = tk.attention_options(q, out, kv_heads=2, scale=c.scale)
    # request 1 of three has no tokens and ends the gap
    tables = torch.cat([c.tables_d[:1], c.tables_d[:1], c.tables_d[1:]]).contiguous()
    lens = torch.tensor([40, 7, 60], dtype=torch.int32, device="cuda")
    view = tk.pool_view(c.pool_d, 0, tables, tables.shape[1])
    for starts, rows in (([4, 14, 14, 44], None), ([-9, 10, 10, 999], None)):
        out.fill_(55), lse.fill_(55)
        if starts[0] == 4:
            q[14:44] = c.q_d[10:]
        room = tk.topkv_attention_workspace_bytes(view, opt, 3, 60)
        work = torch.empty(room, dtype=torch.uint8, device="cuda")
        tk.topkv_attention_prompt(view, opt, 3, lens, torch.tensor(starts, dtype=torch.int32, device="cuda"), 60, q, out, work,
                                  lse=lse)
        if starts[0] == 4:
            assert (out[:4] == 55).all() and (out[44:] == 55).all() and (lse[:4] == 55).all() and (lse[44:] == 55).all()
            c.out_d[:10], c.out_d[10:40] = out[4:14], out[14:44]
            c.lse_d[:10], c.lse_d[10:40] = lse[4:14], lse[14:44]
            c.check()
    torch.cuda.synchronize()


def test_cache_past_32_bits(tk):
    """Pages beyond 4 GiB of a layer."""
    say("[attention] cache past 4 GiB")
    c = Case(19, [300, 40]).device(tk)
    big = torch.empty((1, 80000) + tuple(c.pool_d.shape[2:]), dtype=BF, device="cuda")
    n = c.pool_d.shape[1]
    big[:, 80000 - n:] = c.pool_d
    tables = torch.where(c.tables_d >= 0, c.tables_d + (80000 - n), c.tables_d).contiguous()
    c.cache = tk.pool_view(big, 0, tables, tables.shape[1])
    c.call(tk)
    c.check()
    p = Case(19, [300, 40], [50, 40]).device(tk)
    big[:, 80000 - n:] = p.pool_d
    p.cache = tk.pool_view(big, 0, tables, tables.shape[1])
    p.call(tk)
    p.check()


def test_other_stream(tk):
    say("[attention] another stream")
    c = Case(23, [500, 3000, 41]).device(tk)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    tk.topkv_attention_decode(c.cache, c.options, 3, c.lens_d, c.q_d, c.out_d, c.work, lse=c.lse_d, stream=s)
    s.synchronize()
    c.check()


@pytest.mark.parametrize("decode", [True, False])
def test_captured(tk, decode):
    """A graph replayed over longer and shorter lengths and other queries, eager calls between the replays; two graphs
    that share a workspace, one after the other."""
    say(f"[attention] captured decode={decode}")
    lens = [2000, 10, 333]
    c = Case(29, lens, None if decode else [40, 10, 3]).device(tk)
    c.call(tk)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            tk_call = c.call
            tk_call(tk)
        graphs.append(g)
    rng = np.random.default_rng(3)
    for k in range(6):
        now = [int(rng.integers(0, n + 1)) for n in lens] if k else [0, 0, 0]
        c.lens = now
        c.lens_d.copy_(to_dev(np.array(now, dtype=np.int32)))
        c.out_full.fill_(77), c.lse_d.fill_(77)
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        c.check()
        first = c.out_full.clone()
        c.out_full.fill_(77)
        c.call(tk)
        torch.cuda.synchronize()
        assert torch.equal(first, c.out_full)                     # the same order of sums every time


def test_serving_run(tk):
    """What a decode worker does: unpack prompts into its pool, attend to the last token, branch two beams off, take a page
    for the next token where one is needed, copy, write the token, attend, retire, compact, attend again."""
    say("[attention] serving run")
    H, D, P, G, layers = 2, 64, 16, 4, 2
    lens = [45, 32, 7]
    rows, stride, pages = 6, 4, 30
    g = torch.Generator(device="cuda").manual_seed(1)
    pool = torch.full((layers, pages, 2, P, H, D), float("nan"), dtype=BF, device="cuda")
    tables = torch.full((rows, stride), -1, dtype=torch.int32, device="cuda")
    seq = torch.zeros(rows, dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[[0, 2, 3]] = 1                                            # held by others: a row that is freed later
    tables[5, :3] = torch.tensor([0, 2, 3], dtype=torch.int32)
    seq[5] = 48
    owner = tk.page_owner(refs, tables, seq, page_size=P)
    work = torch.empty(tk.topkv_pages_workspace_bytes(owner), dtype=torch.uint8, device="cuda")
    pairs, result = torch.zeros((pages, 2), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")

    def ints(*v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    tk.topkv_pages_grow(owner, 3, ints(0, 1, 2), ints(*lens), pairs, work, result)
    assert result.tolist() == [0, 0, 6, 0]
    kv = [torch.randn((2, n, H, D), generator=g, device="cuda").to(BF) for n in lens]       # the host's copy of each row
    packed = torch.cat([x.reshape(-1) for x in kv])
    for layer in range(layers):
        tk.topkv_unpack_layer_batched(packed, pool, layer, 3, tables, stride, seq)
    owned = {0: kv[0], 1: kv[1], 2: kv[2]}

    def attend_all(live):
        q = torch.randn((rows, H * G, D), generator=g, device="cuda").to(BF)
        out = torch.zeros_like(q)
        for layer in range(layers):
            view = tk.pool_view(pool, layer, tables, stride)
            opt = tk.attention_options(q, out, kv_heads=H, scale=0.125)
            room = torch.empty(tk.topkv_attention_workspace_bytes(view, opt, rows, rows), dtype=torch.uint8, device="cuda")
            tk.topkv_attention_decode(view, opt, rows, seq, q, out, room)
            for r in live:
                k, v = owned[r][0].double(), owned[r][1].double()
                for h in range(H * G):
                    x = torch.softmax(k[:, h // G] @ q[r, h].double() * 0.125, 0)
                    want, spread = x @ v[:, h // G], x @ v[:, h // G].abs()
                    bound = HALF[BF] * want.abs() + spread * (HALF[BF] + 2.0 ** -15)
                    assert ((out[r, h].double() - want).abs() <= bound).all(), (layer, r, h)

    attend_all([0, 1, 2])
    tk.topkv_pages_fork(owner, 2, ints(0, 0), ints(3, 4), pairs, work, result)
    tk.topkv_copy_pages(pool, pool, 0, layers, pairs, count=result[1:])
    assert result.tolist() == [0, 2, 2, 0]
    owned[3] = owned[4] = kv[0]
    attend_all([0, 1, 2, 3, 4])
    live = ints(0, 1, 2, 3, 4)
    tk.topkv_pages_grow(owner, 5, live, seq[:5] + 1, pairs, work, result)
    tk.topkv_copy_pages(pool, pool, 0, layers, pairs, count=result[1:])
    assert result.tolist() == [0, 0, 1, 0]                          # only the row of 32 tokens needs a page
    new = torch.randn((5, 2, 1, H, D), generator=g, device="cuda").to(BF)
    for layer in range(layers):
        tk.topkv_unpack_layer_window(new, pool, layer, 5, tables, stride, seq, 1)
    for r in range(5):
        owned[r] = torch.cat([owned[r], new[r]], 1)
    attend_all(range(5))
    tk.topkv_pages_free(owner, 2, ints(5, 1), result)
    assert result.tolist() == [0, 0, 6, 0]
    tk.topkv_pages_compact(owner, pairs, work, result)
    tk.topkv_copy_pages(pool, pool, 0, layers, pairs, count=result[1:])
    assert int(result[0]) == 0 and int((refs > 0).sum()) == int(result[2]) and bool((refs[:int(result[2])] > 0).all())
    pool[:, int(result[2]):] = float("nan")                         # the upper part is given away
    attend_all([0, 2, 3, 4])
