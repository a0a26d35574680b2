"""The paged cache on the GPU: block tables against a plain Python statement of the rule, rows in the pages bit for bit,
attention of one token against the formula in 64 bits, and the three as a server runs them."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2601_21896_b200 as pafu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu

T16 = {"bf16": torch.bfloat16, "f16": torch.float16}
POOL = {**T16, "e4m3": torch.float8_e4m3fn}
BAD_PAGE, NO_PAGES = 9, 10


def workspace(cache):
    return torch.zeros(pafu.pafu_paged_workspace_bytes(cache), dtype=torch.uint8, device="cuda")


def header_is_clean(ws):
    return not bool(ws[:12800].any())


def make_pool(n_pages, page, kv, d, dtype, layout, fill):
    shape = (n_pages, page, kv, d) if layout == "tokens" else (n_pages, kv, page, d)
    x = torch.full(shape, fill, device="cuda", dtype=torch.float32).to(dtype)
    return x if layout == "tokens" else x.transpose(1, 2)


class Paged:
    """Pools whose unused places hold NaN, tables whose unused entries are no pages, and the rows of every request."""

    def __init__(self, lens, heads, kv, d, page, layout="tokens", type="bf16", cache="bf16", seed=0, gain=1.0, v_gain=1.0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.lens, self.kv, self.d, self.heads = list(lens), kv, d, heads
        R = len(self.lens)
        count = [-(-n // page) for n in self.lens]
        n_pages, width = sum(count) + 3, max(1, max(count, default=1))
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        table = torch.full((R, width), -1, dtype=torch.int32)
        self.ks = self.vs = None
        if cache == "e4m3":
            self.ks = 0.005 + 0.01 * torch.rand(kv, device="cuda", generator=g)
            self.vs = 0.005 + 0.01 * torch.rand(kv, device="cuda", generator=g)
        K, V = (make_pool(n_pages, page, kv, d, POOL[cache], layout, float("nan")) for _ in range(2))
        self.k, self.v = [], []                       # per request: what the pools hold, [T, kv, d] in 64 bits
        for r, n in enumerate(self.lens):
            table[r, :count[r]] = torch.tensor([order.pop() for _ in range(count[r])], dtype=torch.int32)
            for pool, scale, keep, size in ((K, self.ks, self.k, gain), (V, self.vs, self.v, v_gain)):
                x = torch.randn((n, kv, d), device="cuda", generator=g) * size
                if scale is not None:
                    x = (x / scale[:, None]).clamp(-448, 448)
                x = x.to(POOL[cache])
                t = torch.arange(n, device="cuda")
                at = table[r].long().cuda()[t // page] if n else t
                raw = torch.uint8 if cache == "e4m3" else torch.int16
                pool.view(raw)[at, t % page] = x.view(raw)
                keep.append(x.double() if scale is None else x.double() * scale.double()[:, None])
        self.dtype = T16[type]
        self.Q = torch.randn((R, heads, d), device="cuda", generator=g).to(self.dtype)
        self.len_t = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.table = table.cuda()
        self.cache = pafu.PagedCache(K, V, self.table, heads, dtype=self.dtype, k_scale=self.ks, v_scale=self.vs)
        self.ws = workspace(self.cache)

    def attn(self, sink=0, recent=-1, scale=0.0, ws=None, lens=None):
        R = len(self.lens)
        O = torch.full((R, self.heads, self.d), float("nan"), device="cuda", dtype=self.dtype)
        LSE = torch.full((self.heads, R), float("nan"), device="cuda")
        pafu.pafu_paged_attn(self.cache, self.Q, self.len_t if lens is None else lens, O, LSE, n_sink=sink, n_recent=recent,
                             scale=scale, ws=self.ws if ws is None else ws)
        return O, LSE

    def check(self, O, LSE, sink=0, recent=-1, scale=0.0, lens=None, absent=()):
        """Against the formula in 64 bits.  Bounds, element by element, with w = the softmax weights and s = Q K^T scale:
        rounding the output is eps / 2 of it; a logit is a sum of d exact products in fp32, off by at most
        (d + 8) 2^-23 sum |q k| scale, its scaling and the exponential by 2^-22 (|s| + 2); the probabilities' second term leaves
        2^-17 of them (fp16 products have one term: half a step, 2^-12); n weighted values are added in fp32
        (n 2^-24).  Each of these is a relative error of terms w |v|."""
        scale = scale or 1.0 / math.sqrt(self.d)
        G = self.heads // self.kv
        eps = torch.finfo(self.dtype).eps / 2
        tiny = torch.finfo(self.dtype).tiny
        one_term = self.cache.K.dtype != torch.bfloat16
        for r, n in enumerate(self.lens if lens is None else lens):
            first = 0 if recent < 0 else max(0, n - recent)
            keep = [j for j in list(range(min(sink, first))) + list(range(first, n)) if (r, j) not in absent]
            if not keep:
                assert bool((O[r] == 0).all()) and bool((LSE[:, r] == -math.inf).all()), r
                continue
            t = torch.tensor(keep, device="cuda")
            for h in range(self.kv):
                q = self.Q[r, h * G:(h + 1) * G].double()
                k, v = self.k[r][t, h], self.v[r][t, h]
                s = q @ k.T * scale
                w = torch.softmax(s, -1)
                want, lse = w @ v, torch.logsumexp(s, -1)
                size = (q.abs() @ k.abs().T * scale).amax(-1)
                delta = (self.d + 8) * 2.0 ** -23 * size + 2.0 ** -22 * (s.abs().amax(-1) + 2)
                rel = 2 * delta + (2.0 ** -12 if one_term else 2.0 ** -17) + len(keep) * 2.0 ** -24 + 2.0 ** -21
                tol = eps * want.abs() + rel[:, None] * (w @ v.abs()) * (1 + eps) + tiny
                got = O[r, h * G:(h + 1) * G].double()
                assert bool(torch.isfinite(got).all()), (r, h)
                worst = ((got - want).abs() / tol).max().item()
                assert worst <= 1, (r, h, worst, (got - want).abs().max().item())
                off = (LSE[h * G:(h + 1) * G, r].double() - lse).abs()
                assert bool((off <= delta + 2.0 ** -22 * lse.abs() + len(keep) * 2.0 ** -24 + 2.0 ** -21).all()), (r, h, off.max().item())


EDGE = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 0, 300]


# ------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 2), (12, 1), (20, 1)])
def test_attention_at_every_edge_of_a_tile(cache, type, d, heads, kv):
    x = Paged(EDGE, heads, kv, d, 16, type=type, cache=type if cache == "same" else cache)
    x.check(*x.attn())
    assert header_is_clean(x.ws)


@pytest.mark.parametrize("page", [1, 3, 8, 24, 60, 128, 1560])
@pytest.mark.parametrize("layout", ["tokens", "heads"])
def test_attention_with_pages_of_any_length(page, layout):
    x = Paged([1, 59, 60, 61, 1559, 1560, 1561, 3001], 6, 3, 128, page, layout=layout, seed=page)
    x.check(*x.attn())
    assert header_is_clean(x.ws)


@pytest.mark.parametrize("group", [1, 3, 7, 8, 9, 16, 17, 32, 40])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attention_with_groups_of_any_size(group, cache):
    x = Paged([77, 0, 1000], 2 * group, 2, 128, 16, cache=cache, seed=group)
    x.check(*x.attn())


@pytest.mark.parametrize("sink,recent", [(0, 0), (4, 0), (0, 1), (4, 60), (64, 64), (1, 1000), (1000, 1), (2 ** 40, 2 ** 40), (0, 2 ** 31)])
def test_attention_over_sink_and_recent(sink, recent):
    x = Paged(EDGE, 8, 2, 128, 24, type="f16", cache="f16")
    x.check(*x.attn(sink=sink, recent=recent), sink=sink, recent=recent)


@pytest.mark.parametrize("recent", [-1, -2, -2 ** 31, -2 ** 31 - 1, -2 ** 32, -2 ** 33 + 5, -2 ** 63, 2 ** 63 - 1])
@pytest.mark.parametrize("sink", [0, 2])
def test_any_negative_recent_keeps_every_position(sink, recent):
    """The whole range of n_recent: what its lower 32 bits are does not matter."""
    x = Paged(EDGE, 4, 2, 64, 24)
    x.check(*x.attn(sink=sink, recent=recent), sink=sink, recent=-1)


@pytest.mark.parametrize("d,cache,lens", [(128, "bf16", [20000]), (128, "e4m3", [33333, 1, 5]), (64, "f16", [9999, 10000, 0, 64]), (128, "bf16", [4097] * 9),
                                          (128, "bf16", [150000])])
def test_attention_split_over_the_length(d, cache, lens):
    """Items cut into pieces that many CTAs compute; twice the same bits, counters back at zero."""
    x = Paged(lens, 8, 1, d, 32, type="f16" if cache == "f16" else "bf16", cache=cache, gain=2.0)
    O, LSE = x.attn()
    x.check(O, LSE)
    for _ in range(3):
        O2, LSE2 = x.attn()
        assert torch.equal(O, O2) and torch.equal(LSE, LSE2)
    assert header_is_clean(x.ws)


@pytest.mark.parametrize("d,type,cache,heads,lens", [(128, "bf16", "bf16", 16, [60000]), (64, "f16", "f16", 3, [40000, 2000]),
                                                     (128, "f16", "e4m3", 8, [30000, 30000]), (64, "bf16", "e4m3", 12, [90000])])
def test_pieces_joined_in_groups_repeat_themselves(d, type, cache, heads, lens):
    """Items of more than 16 pieces, whose groups are joined in place of their first piece, up to three levels: what a warp overwrites
    there its lanes have read, so every run gives the same bits."""
    x = Paged(lens, heads, 1, d, 64, type=type, cache=cache, seed=heads)
    O, LSE = x.attn()
    x.check(O, LSE)
    again = [x.attn() for _ in range(60)]
    assert all(torch.equal(O, o) and torch.equal(LSE, s) for o, s in again)
    assert header_is_clean(x.ws)


@pytest.mark.parametrize("n", [600, 3000])
def test_attention_of_many_requests(n):
    """More requests than threads share out, most of them short or empty."""
    g = np.random.default_rng(n)
    lens = [int(v) for v in np.where(g.random(n) < 0.2, 0, g.integers(1, 40, n))]
    x = Paged(lens, 4, 2, 64, 8, seed=n)
    x.check(*x.attn())


@pytest.mark.parametrize("d,type,cache,heads,kv", [(128, "bf16", "bf16", 8, 2), (128, "f16", "e4m3", 3, 3), (128, "bf16", "e4m3", 12, 1),
                                                   (64, "f16", "f16", 20, 1), (64, "bf16", "e4m3", 2, 2), (64, "bf16", "bf16", 40, 2),
                                                   (128, "f16", "f16", 16, 1)])
@pytest.mark.parametrize("sink,recent", [(0, -1), (2, 9)])
def test_attention_of_many_short_items(d, type, cache, heads, kv, sink, recent):
    """Items of at most two tiles, more of them than CTAs: a warp takes them by itself."""
    g = np.random.default_rng(d + heads)
    lens = [int(v) for v in np.where(g.random(700) < 0.1, 0, g.integers(1, 33, 700))]
    x = Paged(lens, heads, kv, d, 8, type=type, cache=cache, seed=heads)
    x.table[3, 0] = -9 if lens[3] else x.table[3, 0]
    x.table[690, 0] = x.cache.n_pages if lens[690] else x.table[690, 0]
    absent = {(r, j) for r in (3, 690) for j in range(8)}
    O, LSE = x.attn(sink=sink, recent=recent)
    x.check(O, LSE, sink=sink, recent=recent, absent=absent)
    O2, LSE2 = x.attn(sink=sink, recent=recent)
    assert torch.equal(O, O2) and torch.equal(LSE, LSE2)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("scale", [1e-3, 0.3, 4.0])
def test_attention_with_peaked_rows(cache, scale):
    """Logits of hundreds, maxima that move from tile to tile; and an explicit scale."""
    x = Paged([700, 65, 3], 4, 2, 128, 16, cache=cache, gain=2.0)
    x.check(*x.attn(scale=scale), scale=scale)


@pytest.mark.parametrize("power", [-100, -20, 60, 110])
def test_attention_of_8_bit_caches_with_queries_beyond_fp16(power):
    """bf16 queries whose size fp16 does not have."""
    x = Paged([200, 40], 4, 2, 128, 16, cache="e4m3")
    x.Q = (x.Q.float() * 2.0 ** power).to(torch.bfloat16)
    scale = 2.0 ** -power / 11.0 if power > -100 else 2.0 ** 100
    x.check(*x.attn(scale=scale), scale=scale)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("lens,kv", [([7000], 1), ([2500] * 40, 16), ([3000, 30] * 30, 12)])
@pytest.mark.parametrize("logit", [5.3, -37.1, 411.0, 20011.0, 100003.0])
def test_sums_do_not_drift_along_a_long_item(logit, lens, kv, type, cache):
    """Keys of one logit, one product each and so exact in fp32, times a factor that is not: sums over any number of tiles are taken relative to
    the same rounded maximum.  The log-sum-exp is the logit plus log n.  Bounds: its two terms and their sum are rounded by 2^-24 each (the logarithm and the
    factors by a few steps more: 2^-21), n equal terms are added in fp32 (n 2^-24); equal values come out as they are, but for
    the sums' rounding, that of one probability (2^-11 for fp16, 2^-17 for bf16) and the output's."""
    d, page = 128, 16
    x = Paged([1] * len(lens), 2 * kv, kv, d, page, type=type, cache=cache)
    count = [-(-n // page) for n in lens]
    width, scale = max(count), 0.7331 * 2.0 ** -3
    # one page serves all: every position holds the same key and the same value
    K, V = (make_pool(1, page, kv, d, POOL[cache], "tokens", 0.0) for _ in range(2))
    K[..., 5], V[..., :] = torch.tensor(64.0).to(POOL[cache]), torch.tensor(1.25).to(POOL[cache])
    table = torch.zeros((len(lens), width), dtype=torch.int32, device="cuda")
    ones = dict(k_scale=torch.ones(kv, device="cuda"), v_scale=torch.ones(kv, device="cuda")) if cache == "e4m3" else {}
    c = pafu.PagedCache(K, V, table, 2 * kv, dtype=x.dtype, **ones)
    Q = torch.zeros((len(lens), 2 * kv, d), device="cuda", dtype=x.dtype)
    Q[..., 5] = logit / (64 * scale)
    O, LSE = torch.full_like(Q, float("nan")), torch.empty((2 * kv, len(lens)), device="cuda")
    pafu.pafu_paged_attn(c, Q, torch.tensor(lens, dtype=torch.int32, device="cuda"), O, LSE, scale=scale, ws=x.ws)
    s = Q[..., 5].double() * 64 * float(torch.tensor(scale, dtype=torch.float32))
    n = torch.tensor(lens, device="cuda").double()[:, None]
    want = (s + torch.log(n)).T
    off = (LSE.double() - want).abs() / (2.0 ** -21 * want.abs() + 2.0 ** -21 * s.abs().T + n.T * 2.0 ** -24 + 2.0 ** -21)
    assert bool((off <= 1).all()), off.max().item()
    eps = torch.finfo(x.dtype).eps / 2
    rel = eps + (2.0 ** -17 if cache == "bf16" else 2.0 ** -11) + max(lens) * 2.0 ** -24 + 2.0 ** -20
    err = (O.double() / 1.25 - 1).abs().max().item()
    assert err <= rel, err


def sink_and_tail(n, margin, spread, d, type, cache, heads, kv, seed=0, sink_at=0, sink_value=0.0):
    """One request of n tokens whose key `sink_at` has a logit of about `margin` above the others', and a value of zero; the others'
    logits are all equal (spread 0) or vary, their values are positive, so that what is lost of their weights does not cancel."""
    x = Paged([n], heads, kv, d, 16, type=type, cache=cache, seed=seed)
    g = torch.Generator("cuda").manual_seed(seed + 1)
    k = torch.randn((n, kv, d), device="cuda", generator=g) * spread
    k[..., 0] = 0.0
    k[sink_at] = 0.0
    k[sink_at, :, 0] = margin * math.sqrt(d) / 128.0
    v = torch.rand((n, kv, d), device="cuda", generator=g) + 0.5
    v[sink_at] = sink_value
    x.Q[..., 0] = 128.0
    t = torch.arange(n, device="cuda")
    at = x.table[0].long()[t // 16]
    for pool, scale, keep, new in ((x.cache.K, x.ks, x.k, k), (x.cache.V, x.vs, x.v, v)):
        new = (new if scale is None else (new / scale[:, None]).clamp(-448, 448)).to(POOL[cache])
        raw = torch.uint8 if cache == "e4m3" else torch.int16
        pool.view(raw)[at, t % 16] = new.view(raw)
        keep[0] = new.double() if scale is None else new.double() * scale.double()[:, None]
    return x


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("n,spread,d,heads,kv", [(40, 0.0, 64, 4, 1), (300, 0.0, 128, 3, 3), (2000, 0.0, 128, 8, 1), (2000, 1.0, 64, 16, 1),
                                                 (20000, 0.5, 128, 4, 2), (100000, 1.0, 128, 4, 1)])
@pytest.mark.parametrize("margin", [8, 12, 16, 20])
def test_small_probabilities_beside_a_sink(margin, n, spread, d, heads, kv, type, cache):
    """A first token that draws the attention while its value is nothing: the output is the others', whose probabilities are e^-8 to e^-20 of
    the largest.  Bound: as in Paged.check, with the probabilities' rounding as the format has it.  fp16 rounds p 2^15 (p <= 1) by at
    most 2^-11 of it, or 2^-25 where that is a subnormal: 2^-40 of the largest probability.  bf16 leaves 2^-17 after its second term."""
    x = sink_and_tail(n, margin, spread, d, type, cache, heads, kv, seed=n + margin)
    O, LSE = x.attn()
    G, scale, eps = heads // kv, 1.0 / math.sqrt(d), torch.finfo(x.dtype).eps / 2
    one_term = cache != "bf16"
    for h in range(kv):
        q, k, v = x.Q[0, h * G:(h + 1) * G].double(), x.k[0][:, h], x.v[0][:, h]
        s = q @ k.T * scale
        w = torch.softmax(s, -1)
        want, lse = w @ v, torch.logsumexp(s, -1)
        assert bool((s[:, 0] - s[:, 1:].mean(-1) > 0.85 * margin).all())                    # the keys' own rounding included
        size = (q.abs() @ k.abs().T * scale).amax(-1)
        delta = (d + 8) * 2.0 ** -23 * size + 2.0 ** -22 * (s.abs().amax(-1) + 2)
        rel = 2 * delta + (2.0 ** -11 if one_term else 2.0 ** -17) + n * 2.0 ** -24 + 2.0 ** -21
        lost = 2.0 ** -40 * w.amax(-1, keepdim=True) * v.sum(0) if one_term else 0.0
        tol = eps * want.abs() + rel[:, None] * want * (1 + eps) + lost + torch.finfo(x.dtype).smallest_normal * eps
        got = O[0, h * G:(h + 1) * G].double()
        worst = ((got - want).abs() / tol).max().item()
        assert worst <= 1, (h, worst, ((got - want).abs() / want).max().item())
        off = (LSE[h * G:(h + 1) * G, 0].double() - lse).abs()
        assert bool((off <= delta + 2.0 ** -22 * lse.abs() + n * 2.0 ** -24 + 2.0 ** -21).all()), (h, off.max().item())


def test_small_probabilities_of_many_short_items():
    """The same for items that a warp takes by itself, and for a sink that comes last: what is already summed is scaled down."""
    for sink_at in (0, 29):
        x = sink_and_tail(30, 16, 0.0, 128, "f16", "f16", 2, 1, sink_at=sink_at)
        one, one_lse = x.attn()
        many = 400
        table = x.table.repeat(many, 1)
        cache = pafu.PagedCache(x.cache.K, x.cache.V, table, 2)
        Q, lens = x.Q.repeat(many, 1, 1), x.len_t.repeat(many)
        O, LSE = torch.empty_like(Q), torch.empty((2, many), device="cuda")
        pafu.pafu_paged_attn(cache, Q, lens, O, LSE, ws=x.ws)
        s = x.Q[0].double() @ x.k[0][:, 0].T / math.sqrt(128)
        want, lse = torch.softmax(s, -1) @ x.v[0][:, 0], torch.logsumexp(s, -1)
        for o, l in ((one, one_lse), (O, LSE)):
            # one rounding each of probabilities and output, 2^-11; the logit of the sink, 136 products of up to 16 in all, and its exponential
            # by 2^-18; twice the smallest step of an output
            assert bool(((o.double() - want).abs() <= (2 * 2.0 ** -11 + 2 * 136 * 2.0 ** -23 * 16 + 2.0 ** -16) * want + 2.0 ** -24).all())
            assert bool(((l.double() - lse[:, None]).abs() <= 136 * 2.0 ** -23 * 16 + 2.0 ** -17).all())


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("n,sink_at", [(20, 3), (500, 0), (500, 499), (5000, 2500)])
@pytest.mark.parametrize("size", [10, 20, 24, 28, 30])
def test_huge_logits_leave_the_largest(size, n, sink_at, type, cache):
    """A largest logit of about 2^size, which fp32 holds to whole numbers and less: the output is that key's value, and what rounding the
    maximum leaves over cancels or does not arise.  The probability and the output are rounded by at most 2^-11 and eps / 2; the other keys' logits lie a
    fifth of 2^size and more below and count for nothing."""
    x = sink_and_tail(n, 20, 0.5, 128, type, cache, 4, 2, seed=n, sink_at=sink_at, sink_value=1.3125)
    scale = 2.0 ** size / (20 * math.sqrt(128))
    O, LSE = x.attn(scale=scale)
    eps = torch.finfo(x.dtype).eps / 2
    for h in range(2):
        s = x.Q[0, 2 * h:2 * h + 2].double() @ x.k[0][:, h].T * float(torch.tensor(scale, dtype=torch.float32))
        two = s.topk(2).values
        assert bool((s.argmax(-1) == sink_at).all()) and bool((two[:, 0] - two[:, 1] > 0.2 * 2.0 ** size).all())
        want = x.v[0][sink_at, h]
        got = O[0, 2 * h:2 * h + 2].double()
        assert bool(((got - want).abs() <= (eps + 2.0 ** -11 + 2.0 ** -20) * want.abs()).all()), (got - want).abs().max()
        # the logit: its factor, its products' sum and their product are rounded, 136 steps of 2^-23 at most
        assert bool(((LSE[2 * h:2 * h + 2, 0].double() - two[:, 0]).abs() <= 140 * 2.0 ** -23 * two[:, 0]).all())


def test_attention_reads_strided_queries_and_pools():
    """Queries inside fused rows; K and V inside one tensor, heads not contiguous."""
    x = Paged([130, 33], 6, 3, 128, 16)
    fused = torch.full((2, 12, 128), float("nan"), device="cuda", dtype=x.dtype)
    fused[:, 2:8] = x.Q
    both = torch.full((x.cache.n_pages, 16, 3, 2, 128), float("nan"), device="cuda", dtype=x.dtype)
    both[..., 0, :], both[..., 1, :] = x.cache.K, x.cache.V
    O, LSE = x.attn()
    x.cache = pafu.PagedCache(both[..., 0, :], both[..., 1, :], x.table, 6)
    x.Q = fused[:, 2:8]
    O2, LSE2 = x.attn()
    x.check(O2, LSE2)
    assert torch.equal(O, O2) and torch.equal(LSE, LSE2)


def test_attention_leaves_out_what_is_no_page_and_cuts_lengths():
    x = Paged([100, 200, 50], 4, 2, 64, 16)
    x.table[1, 3] = x.cache.n_pages                      # request 1, tokens 48 to 63
    x.table[2, 0] = -7                                   # request 2, tokens 0 to 15
    absent = {(1, j) for j in range(48, 64)} | {(2, j) for j in range(16)}
    x.check(*x.attn(), absent=absent)
    assert pafu.pafu_workspace_status(x.ws) == BAD_PAGE
    x.ws[:256] = 0
    lens = torch.tensor([100, -5, 10 ** 6], dtype=torch.int32, device="cuda")
    O, LSE = x.attn(lens=lens)
    assert pafu.pafu_workspace_status(x.ws) == BAD_PAGE
    x.check(O[:2], LSE[:, :2], lens=[100, 0], absent=absent)
    # cut to the table's 208 tokens, request 2 reads all of its four pages, and so the NaN behind its 50 tokens
    assert bool(torch.isnan(O[2]).all()) and bool(torch.isnan(LSE[:, 2]).all())


def test_attention_addresses_past_32_bits():
    """A pool of more than 4 GiB, and more than 2^31 elements: the last pages are as good as the first."""
    n_pages, page, kv, d = 70000, 64, 4, 128
    K = torch.zeros((n_pages, page, kv, d), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    assert K.numel() > 2 ** 31 and K.numel() * 2 > 2 ** 32
    x = Paged([200, 130], 4, 4, d, page)
    where = torch.tensor([[n_pages - 1, 1, n_pages - 2, 65536], [n_pages - 3, 32767, 32768, 5]], dtype=torch.int32, device="cuda")
    for r in range(2):
        for i in range(-(-x.lens[r] // page)):
            K[int(where[r, i])], V[int(where[r, i])] = x.cache.K[int(x.table[r, i])], x.cache.V[int(x.table[r, i])]
    O, LSE = x.attn()
    x.cache = pafu.PagedCache(K, V, where, 4)
    O2, LSE2 = x.attn()
    assert torch.equal(O, O2) and torch.equal(LSE, LSE2)
    # rows written there, too
    slots = torch.tensor([int(where[0, 0]) * page + 63, -1], device="cuda")
    new = torch.randn((2, kv, d), device="cuda").to(torch.bfloat16)
    pafu.pafu_paged_append(x.cache, new, new, slots, ws=x.ws)
    assert torch.equal(K[n_pages - 1, 63], new[0]) and torch.equal(V[n_pages - 1, 63], new[0])


def test_attention_captured_once_follows_lengths_and_tables():
    x = Paged([900, 40, 0, 333], 8, 2, 128, 16)
    O = torch.empty((4, 8, 128), device="cuda", dtype=x.dtype)
    LSE = torch.empty((8, 4), device="cuda")
    call = lambda: pafu.pafu_paged_attn(x.cache, x.Q, x.len_t, O, LSE, ws=x.ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens in ([900, 40, 0, 333], [1, 0, 0, 332], [0, 0, 0, 0], [899, 17, 0, 1]):
        x.len_t.copy_(torch.tensor(lens, dtype=torch.int32))
        O.fill_(float("nan"))
        LSE.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        x.check(O, LSE, lens=lens)
    assert header_is_clean(x.ws)


def test_first_calls_of_a_process_inside_a_capture():
    """Nothing that the first launch of a kernel sets up is forbidden while a stream is captured."""
    code = """
import sys; sys.path.insert(0, %r)
import torch
import tests.test_paged_gpu as T
x = T.Paged([100, 3], 4, 2, 64, 16)
t = T.Tables(2, 4, 8, 10)
n = T.Paged([4], 2, 2, 128, 4, cache="e4m3")
new = torch.ones((1, 2, 128), device="cuda", dtype=torch.bfloat16)
slots = torch.tensor([0], device="cuda")
O, LSE = torch.empty_like(x.Q), torch.empty((4, 2), device="cuda")
out = [torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda"),
       torch.empty(3, dtype=torch.int64, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")]
after = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    T.pafu.pafu_paged_tables(t.cache, t.lens, after, t.f, t.nf, out[0], out[1], out[2], out[3], ws=t.ws)
    T.pafu.pafu_paged_append(n.cache, new, new, slots, ws=n.ws)
    T.pafu.pafu_paged_attn(x.cache, x.Q, x.len_t, O, LSE, ws=x.ws)
g.replay()
torch.cuda.synchronize()
x.check(O, LSE)
assert out[1].tolist() == [1, 2] and int(out[0]) == 8 and (out[2] >= 0).all()
print("fine")
""" % ROOT
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("captured", [False, True])
def test_attention_sees_rows_written_just_ahead(captured):
    """Rows of the same places written over and over, the attention launched right behind each time: it has read the new ones."""
    lens = [64, 1, 40]
    x = Paged(lens, 4, 2, 128, 16)
    places = [[int(x.table[r, t // 16]) * 16 + t % 16 for t in range(n)] for r, n in enumerate(lens)]
    slots = torch.tensor(sum(places, []), device="cuda")
    rows = torch.randn((30, 2, len(slots), 2, 128), device="cuda").to(torch.bfloat16)
    outs = [(torch.empty_like(x.Q), torch.empty((4, 3), device="cuda")) for _ in rows]

    def steps():
        for (k, v), (O, LSE) in zip(rows, outs):
            pafu.pafu_paged_append(x.cache, k, v, slots, ws=x.ws)
            pafu.pafu_paged_attn(x.cache, x.Q, x.len_t, O, LSE, ws=x.ws)

    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            steps()
        graph.replay()
    else:
        steps()
    torch.cuda.synchronize()
    for (k, v), (O, LSE) in zip(rows, outs):
        x.k, x.v = list(k.double().split(lens)), list(v.double().split(lens))
        x.check(O, LSE)


def test_a_workspace_serves_one_cache_after_the_other():
    a, b = Paged([3000, 7], 8, 1, 128, 16, seed=1), Paged([2000] * 3, 4, 2, 64, 8, seed=2)
    for _ in range(3):
        for x in (a, b):
            x.check(*x.attn(ws=a.ws))


def test_two_streams_with_a_workspace_each():
    a, b = Paged([5000, 10], 8, 1, 128, 16, seed=1), Paged([7000], 8, 1, 128, 16, seed=2)
    want = a.attn() + b.attn()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i, x in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(x.attn())
    torch.cuda.synchronize()
    for i in range(2):
        for O, LSE in got[i]:
            assert torch.equal(O, want[2 * i]) and torch.equal(LSE, want[2 * i + 1])


def test_attention_agrees_with_chunk_attention():
    """One query of the chunk kernel over the same keys in one buffer."""
    N, D, T = 12, 128, 1000
    x = Paged([T], N, N, D, 60)
    O, LSE = x.attn()
    shape = pafu.Shape(N, D, None, [0, 1])
    O2, LSE2 = torch.empty_like(O), torch.empty_like(LSE)
    ws = torch.zeros(pafu.pafu_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    K, V = x.k[0].to(torch.bfloat16), x.v[0].to(torch.bfloat16)
    pafu.pafu_chunk_attn(x.Q, K, V, [0, T], None, None, shape, 0.0, O2, LSE2, ws)
    # each is within 2^-8 of |o| and the chunk kernel's probabilities within 2^-8 of theirs
    assert (O.float() - O2.float()).abs().max() <= 3 * 2.0 ** -8 * (x.v[0].abs().max().item())
    assert (LSE - LSE2).abs().max() <= 1e-4


# ------------------------------------------------------------------------------------ append
def e4m3_values():
    """The non-negative finite e4m3 values, from the format: 4 exponent bits (bias 7), 3 mantissa bits."""
    return np.array([m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)
                                                             if not (e == 15 and m == 7)])


def nearest_e4m3(x):
    """The nearest e4m3 values to a float64 tensor's, ties to even, beyond 448 to 448."""
    grid = torch.from_numpy(e4m3_values()).to(x.device)
    a = x.abs().clamp(max=448.0)
    up = torch.searchsorted(grid, a).clamp(1, len(grid) - 1)
    lo, hi = grid[up - 1], grid[up]
    upper = (hi - a < a - lo) | ((hi - a == a - lo) & (up % 2 == 0))
    return torch.where(upper, hi, lo) * torch.sign(x)


def test_append_rounds_next_to_a_border():
    """Quotients a few parts in 10^8 beside a border between two e4m3 values, which a quotient rounded to fp32 no longer tells apart;
    and quotients on one."""
    base = e4m3_values()
    borders = (base[1:] + base[:-1]) / 2
    scales, rows = [], []
    rng = np.random.default_rng(0)
    for h in range(40):
        b = float(rng.choice(borders[4:]))
        x = np.float64(np.float16(rng.uniform(0.5, 4.0)))                # the row's value; the scale is next to x / border
        s = np.nextafter(np.float32(x / b), np.float32(rng.choice([0.0, 10.0]))) if h % 4 else np.float32(x / b)
        scales.append(s)
        rows.append(np.concatenate([x * 2.0 ** np.arange(-6, 6), -x * 2.0 ** np.arange(-6, 6)]))
    kv, d = 40, 64
    K, V = (make_pool(1, 1, kv, d, torch.float8_e4m3fn, "tokens", 1.0) for _ in range(2))
    ks = torch.tensor(np.array(scales, dtype=np.float32), device="cuda")
    cache = pafu.PagedCache(K, V, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), kv, dtype=torch.float16, k_scale=ks, v_scale=ks)
    x = torch.zeros((1, kv, d), device="cuda", dtype=torch.float16)
    x[0, :, :24] = torch.from_numpy(np.array(rows)).to("cuda").half()
    pafu.pafu_paged_append(cache, x, -x, torch.tensor([0], device="cuda"), ws=workspace(cache))
    want = nearest_e4m3(x[0].double() / ks.double()[:, None])
    assert torch.equal(K[0, 0].double(), want) and torch.equal(V[0, 0].double(), -want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["tokens", "heads"])
@pytest.mark.parametrize("n,kv,page", [(1, 1, 1), (5, 3, 16), (257, 2, 60), (1000, 12, 7)])
@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_append_copies_rows(type, n, kv, page, layout, d):
    n_pages = n // page + 3
    K, V = (make_pool(n_pages, page, kv, d, T16[type], layout, 7.0) for _ in range(2))
    cache = pafu.PagedCache(K, V, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), kv)
    ws = workspace(cache)
    g = torch.Generator("cuda").manual_seed(n)
    rows = torch.randint(-2 ** 15, 2 ** 15, (n, 3 * kv, d), device="cuda", generator=g, dtype=torch.int32).to(torch.int16)
    Kn, Vn = rows[:, kv:2 * kv].view(T16[type]), rows[:, 2 * kv:].view(T16[type])       # any bits: NaN, infinities, subnormals
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(n))[:n].cuda()
    slots[n // 2] = -1
    if n > 4:
        slots[-2:] = torch.tensor([-1, -2 ** 62])
    want_K, want_V = K.clone(), V.clone()
    live = (slots >= 0).nonzero()[:, 0]
    for want, new in ((want_K, Kn), (want_V, Vn)):
        want.view(torch.int16)[slots[live] // page, slots[live] % page] = new.view(torch.int16)[live]
    pafu.pafu_paged_append(cache, Kn, Vn, slots, ws=ws)
    assert torch.equal(K.view(torch.int16), want_K.view(torch.int16)) and torch.equal(V.view(torch.int16), want_V.view(torch.int16))
    assert header_is_clean(ws)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("scaled", [True, False])
def test_append_rounds_to_8_bits(type, scaled, d):
    n, kv, page = 300, 3, 16
    K, V = (make_pool(24, page, kv, d, torch.float8_e4m3fn, "tokens", 1.0) for _ in range(2))
    g = torch.Generator("cuda").manual_seed(5)
    ks = vs = None
    if scaled:
        ks, vs = 0.01 + torch.rand(kv, device="cuda", generator=g), 0.01 + torch.rand(kv, device="cuda", generator=g)
    cache = pafu.PagedCache(K, V, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), kv, dtype=T16[type], k_scale=ks, v_scale=vs)
    x = [torch.randn((n, kv, d), device="cuda", generator=g) * 2.0 ** torch.randint(-12, 9, (n, 1, 1), device="cuda", generator=g)
         for _ in range(2)]
    x = [v.to(T16[type]) for v in x]
    special = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, 448, 449, -463, 464, 480, 1e4, 2.0 ** -10, 2.0 ** -9, 3 * 2.0 ** -10,
                            1.0625, 1.1875, -1.0625, 17, 19, 0.0009765625], device="cuda").to(T16[type])
    for v in x:
        v[0, :, :len(special)] = special
    slots = torch.randperm(24 * page, generator=torch.Generator().manual_seed(1))[:n].cuda()
    pafu.pafu_paged_append(cache, x[0], x[1], slots, ws=workspace(cache))
    grid = e4m3_values()
    for pool, v, s in ((K, x[0], ks), (V, x[1], vs)):
        got = pool.double()[slots // page, slots % page].cpu().numpy()
        q = (v.double() if s is None else v.double() / s.double()[:, None]).cpu().numpy()
        nan = np.isnan(q)
        assert np.array_equal(np.isnan(got), nan)
        q, got = np.clip(q[~nan], -448, 448), got[~nan]
        # the nearest value to the quotient, which 64 bits hold to 2^-53
        up = np.clip(np.searchsorted(grid, np.abs(q)), 1, len(grid) - 1)
        nearest = np.minimum(np.abs(grid[up] - np.abs(q)), np.abs(np.abs(q) - grid[up - 1]))
        assert np.all(np.abs(got - q) <= nearest + 2.0 ** -50 * np.abs(q))
        assert np.all(np.signbit(got) == np.signbit(q))
        if s is None:                              # ties to the even mantissa
            tie = np.abs(np.abs(grid[up] - np.abs(q)) - np.abs(np.abs(q) - grid[up - 1])) == 0
            even = np.where((up % 2) == 0, grid[up], grid[up - 1])
            assert tie.any() and np.array_equal(np.abs(got[tie]), even[tie])


def test_append_leaves_out_slots_past_the_pool():
    K, V = (make_pool(2, 16, 1, 64, torch.bfloat16, "tokens", 3.0) for _ in range(2))
    cache = pafu.PagedCache(K, V, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), 1)
    ws = workspace(cache)
    new = torch.ones((3, 1, 64), device="cuda", dtype=torch.bfloat16)
    pafu.pafu_paged_append(cache, new, new, torch.tensor([32, 2 ** 40, 31], device="cuda"), ws=ws)
    assert pafu.pafu_workspace_status(ws) == BAD_PAGE
    assert bool((K[1, 15] == 1).all()) and bool((K.reshape(32, 64)[:31] == 3).all())


# ------------------------------------------------------------------------------------ tables
def plain_tables(page, old, new, table, free, n_free, n_slots, n_pages):
    """The rule, request by request.  None where nothing may change hands."""
    W = table.shape[1]
    P = lambda n: -(-n // page)
    if any(n < 0 for n in old + new) or any(P(n) > W for n in old + new) or not 0 <= n_free <= n_pages:
        return BAD_PAGE
    table, stack = table.copy(), list(free[:n_free])
    for r in range(len(old)):
        stack += [int(p) for p in table[r, P(new[r]):P(old[r])]]
    if sum(max(P(n) - P(o), 0) for o, n in zip(old, new)) > len(stack) or sum(max(n - o, 0) for o, n in zip(old, new)) > n_slots:
        return NO_PAGES
    slots, cu = [], [0]
    for r in range(len(old)):
        for c in range(P(old[r]), P(new[r])):
            table[r, c] = stack.pop()
        slots += [int(table[r, t // page]) * page + t % page for t in range(old[r], new[r])]
        cu.append(len(slots))
    out = free.copy()
    out[n_free:len(stack)] = stack[n_free:]
    return table, out, len(stack), slots + [-1] * (n_slots - len(slots)), cu


class Tables:
    def __init__(self, R, width, page, n_pages, seed=0):
        rng = np.random.default_rng(seed)
        self.rng, self.R, self.page, self.n_pages = rng, R, page, n_pages
        self.table = rng.integers(-5, 5, (R, width)).astype(np.int32)          # entries behind a request's pages mean nothing
        self.free, self.n_free = rng.permutation(n_pages).astype(np.int32), n_pages
        self.t = torch.from_numpy(self.table.copy()).cuda()
        self.f = torch.from_numpy(self.free.copy()).cuda()
        self.nf = torch.tensor([n_pages], dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(R, dtype=torch.int32, device="cuda")
        pool = torch.zeros((n_pages, page, 1, 64), dtype=torch.bfloat16, device="cuda")
        self.cache = pafu.PagedCache(pool, pool, self.t, 1)
        self.ws = workspace(self.cache)

    def step(self, new, n_slots, in_place=True):
        old = self.lens.tolist()
        want = plain_tables(self.page, old, new, self.table, self.free, self.n_free, n_slots, self.n_pages)
        slots = torch.full((n_slots,), 99, dtype=torch.int64, device="cuda")
        cu = torch.full((self.R + 1,), 99, dtype=torch.int32, device="cuda")
        lens_out = self.lens if in_place else torch.empty_like(self.lens)
        nf_out = self.nf if in_place else torch.empty_like(self.nf)
        pafu.pafu_paged_tables(self.cache, self.lens, torch.tensor(new, dtype=torch.int32, device="cuda"), self.f, self.nf, nf_out,
                               lens_out, slots, cu, ws=self.ws)
        status = pafu.pafu_workspace_status(self.ws)
        if isinstance(want, int):
            assert status == want
            self.ws[:256] = 0
            assert lens_out.tolist() == old and int(nf_out) == self.n_free and slots.tolist() == [-1] * n_slots
            assert cu.tolist() == [0] * (self.R + 1)
        else:
            assert status == 0
            self.table, self.free, self.n_free, want_slots, want_cu = want
            assert lens_out.tolist() == new and int(nf_out) == self.n_free
            assert slots.tolist() == want_slots and cu.tolist() == want_cu
        assert np.array_equal(self.t.cpu().numpy(), self.table) and np.array_equal(self.f.cpu().numpy(), self.free)
        assert header_is_clean(self.ws)
        self.lens, self.nf = lens_out, nf_out
        return not isinstance(want, int)


@pytest.mark.parametrize("R,page,in_place", [(1, 1, True), (3, 16, False), (40, 7, True), (513, 16, True), (1500, 5, False)])
def test_tables_over_many_steps(R, page, in_place):
    """Requests begin, grow, take tokens back and end; the pool runs dry now and then."""
    width = 12
    x = Tables(R, width, page, max(4, R * width // 3), seed=R)
    did = []
    for step in range(14):
        old = x.lens.tolist()
        kind = x.rng.random(R)
        new = [min(width * page, o + 1) if k < 0.5 else int(x.rng.integers(0, width * page + 1)) if k < 0.65 else 0 if k < 0.8
               else max(0, o - int(x.rng.integers(0, 9))) if k < 0.9 else o for o, k in zip(old, kind)]
        total = sum(max(n - o, 0) for o, n in zip(old, new))
        did.append(x.step(new, total + int(x.rng.integers(0, 50)), in_place))
    assert any(did)


def test_tables_refuse_as_a_whole():
    x = Tables(4, 4, 8, 10, seed=1)
    assert x.step([20, 8, 0, 1], 29)                    # 3 + 1 + 0 + 1 pages
    assert not x.step([32, 32, 9, 1], 100)              # 4 + 4 + 2 + 1 pages: one too few
    assert not x.step([21, 8, 0, 1], 0)                 # no place in the slot map
    assert not x.step([20, -1, 0, 1], 5)
    assert not x.step([20, 33, 0, 1], 50)               # more than the table is wide
    assert x.step([0, 32, 8, 1], 40)                    # with the pages that request 0 gives back
    assert x.step([0, 0, 0, 0], 0)
    assert x.n_free == 10
    keep, x.nf = x.nf, torch.tensor([11], dtype=torch.int32, device="cuda")
    x.n_free = 11
    assert not x.step([1, 1, 1, 1], 4)
    x.n_free, x.nf = 10, keep
    assert x.step([32, 0, 32, 9], 73)                   # to the last page
    assert x.n_free == 0


@pytest.mark.parametrize("bad", [-1, -2 ** 31, 40, 2 ** 31 - 1])
@pytest.mark.parametrize("where", ["partly filled", "popped", "given back", "given back and taken"])
def test_tables_report_what_is_no_page(where, bad):
    """A table entry or free-list entry that is no page of the pool is handed on as it stands, its new tokens get no slot, and it is
    reported: a lost row never looks like padding."""
    n_pages, page, R, width = 40, 8, 3, 6
    x = Tables(R, width, page, n_pages)
    assert x.step([13, 20, 9], 42)                                        # two, three and two pages
    table, free, n_free = x.table.copy(), x.free.copy(), x.n_free
    if where == "partly filled":
        table[0, 1], new = bad, [15, 21, 9]
    elif where == "popped":
        free[n_free - 1], new = bad, [13, 26, 9]                          # request 1 goes on to a new page
    elif where == "given back":
        table[2, 0], new = bad, [14, 21, 0]
    else:
        table[2, 1], new = bad, [14, 26, 0]                               # request 2's last page is request 1's next one
    x.t.copy_(torch.from_numpy(table))
    x.f.copy_(torch.from_numpy(free))
    want = plain_tables(page, [13, 20, 9], new, table, free, n_free, 12, n_pages)
    slots, cu = torch.full((12,), 99, dtype=torch.int64, device="cuda"), torch.empty(R + 1, dtype=torch.int32, device="cuda")
    pafu.pafu_paged_tables(x.cache, x.lens, torch.tensor(new, dtype=torch.int32, device="cuda"), x.f, x.nf, x.nf, x.lens, slots, cu, ws=x.ws)
    assert pafu.pafu_workspace_status(x.ws) == BAD_PAGE
    assert x.lens.tolist() == new and int(x.nf) == want[2] and cu.tolist() == want[4]
    assert np.array_equal(x.t.cpu().numpy(), want[0]) and np.array_equal(x.f.cpu().numpy(), want[1])
    assert slots.tolist() == [s if 0 <= s < n_pages * page else -1 for s in want[3]]
    assert not bool(x.ws[256:12800].any())


def test_tables_of_a_long_step():
    """More new tokens than a CTA takes; pages of one request given to another in the same step."""
    x = Tables(6, 3000, 16, 3200, seed=3)
    assert x.step([40000, 5, 0, 0, 9000, 1], 50000)
    assert x.step([0, 30000, 1, 17, 9001, 2], 40000)
    assert x.step([3, 0, 48000, 0, 100, 2], 60001)


def test_tables_without_requests():
    x = Tables(0, 4, 8, 10)
    assert x.step([], 3) and x.step([], 0)


# ------------------------------------------------------------------------------------ a server's steps
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("captured", [False, True])
def test_steps_of_a_server(cache, captured):
    """Tables, rows and attention for steps on end, two layers, prompts of any length, requests that end: what the attention
    sees is what was written.  Captured: one graph of the step, replayed with other lengths."""
    R, heads, kv, d, page, width, n_pages, cap = 5, 8, 2, 64, 8, 40, 120, 400
    rng = np.random.default_rng(3)
    gen = torch.Generator("cuda").manual_seed(3)
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    scale = dict(k_scale=torch.full((kv,), 0.02, device="cuda"), v_scale=torch.full((kv,), 0.03, device="cuda")) if cache == "e4m3" else {}
    caches = [pafu.PagedCache(make_pool(n_pages, page, kv, d, POOL[cache], "heads", float("nan")),
                              make_pool(n_pages, page, kv, d, POOL[cache], "heads", float("nan")), table, heads,
                              dtype=torch.bfloat16, **scale) for _ in range(2)]
    ws = workspace(caches[0])
    lens, target = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
    free, n_free = torch.arange(n_pages, dtype=torch.int32, device="cuda"), torch.tensor([n_pages], dtype=torch.int32, device="cuda")
    slots, cu = torch.empty(cap, dtype=torch.int64, device="cuda"), torch.empty(R + 1, dtype=torch.int32, device="cuda")
    rows = [torch.empty((cap, heads + 2 * kv, d), device="cuda", dtype=torch.bfloat16) for _ in caches]
    Q = torch.empty((R, heads, d), device="cuda", dtype=torch.bfloat16)
    O = [torch.empty_like(Q) for _ in caches]
    LSE = [torch.empty((heads, R), device="cuda") for _ in caches]

    def step():
        pafu.pafu_paged_tables(caches[0], lens, target, free, n_free, n_free, lens, slots, cu, ws=ws)
        for i, c in enumerate(caches):
            pafu.pafu_paged_append(c, rows[i][:, heads:heads + kv], rows[i][:, heads + kv:], slots, ws=ws)
            pafu.pafu_paged_attn(c, Q, lens, O[i], LSE[i], ws=ws)

    run = step
    if captured:
        step()                                         # lengths 0 to 0: nothing changes
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    held = [[[[] for _ in range(2)] for _ in range(R)] for _ in caches]      # [layer][request][K, V]: rows in order
    now = [0] * R
    for it in range(12):
        new = [0 if n and rng.random() < 0.15 else int(rng.integers(1, 70)) if n == 0 and rng.random() < 0.7 else n + 1 if n else 0 for n in now]
        for i in range(2):
            rows[i].copy_(torch.randn(rows[i].shape, device="cuda", generator=gen))
        Q.copy_(torch.randn(Q.shape, device="cuda", generator=gen))
        target.copy_(torch.tensor(new, dtype=torch.int32))
        run()
        assert pafu.pafu_workspace_status(ws) == 0
        at = 0
        for r in range(R):
            grown = max(new[r] - now[r], 0)
            for i in range(2):
                for kind in range(2):
                    x = rows[i][at:at + grown, heads + kind * kv: heads + (kind + 1) * kv].double()
                    if cache == "e4m3":
                        s = (0.02, 0.03)[kind]
                        s = float(torch.tensor(s, dtype=torch.float32))
                        x = nearest_e4m3(x / s) * s
                    held[i][r][kind] = (held[i][r][kind] if now[r] and new[r] else []) + [x]
            at += grown
        now = new
        for i in range(2):
            p = Paged.__new__(Paged)
            p.lens, p.kv, p.d, p.heads, p.dtype, p.cache, p.Q = now, kv, d, heads, torch.bfloat16, caches[i], Q
            p.k = [torch.cat(h[0])[:n] for h, n in zip(held[i], now)]
            p.v = [torch.cat(h[1])[:n] for h, n in zip(held[i], now)]
            p.check(O[i], LSE[i])
    assert max(now) > 0 and header_is_clean(ws)


def test_steps_refuse_tensors_of_the_wrong_kind():
    x = Paged([20, 3], 4, 2, 64, 16)
    O, LSE = x.attn()
    bad = [dict(Q=x.Q.float()), dict(Q=x.Q[:1]), dict(lens=x.len_t.long()), dict(O=O[:, :2]), dict(LSE=LSE.double()),
           dict(lens=x.len_t.cpu())]
    for b in bad:
        a = dict(Q=x.Q, lens=x.len_t, O=O, LSE=LSE)
        a.update(b)
        with pytest.raises(pafu.PafuError) as e:
            pafu.pafu_paged_attn(x.cache, a["Q"], a["lens"], a["O"], a["LSE"], ws=x.ws)
        assert e.value.status == 1
    with pytest.raises(pafu.PafuError):
        pafu.pafu_paged_append(x.cache, x.Q[:, :2].float(), x.Q[:, :2].float(), x.len_t.long(), ws=x.ws)
    with pytest.raises(pafu.PafuError):
        pafu.pafu_paged_attn(x.cache, x.Q, x.len_t, x.Q, LSE, ws=x.ws)                  # output over input
