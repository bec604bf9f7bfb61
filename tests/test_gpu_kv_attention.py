"""gmlp_kv_attention against its definition in 64 bits: lengths, chunks, heads, pages, ragged batches, masks, numbers that are no numbers in
places that are not seen, bad tables, large caches, streams and graphs."""
import math

import pytest
import torch

import _paged as P
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def bf16(seed, *shape):
    return torch.randn(*shape, generator=gen(seed), device=DEV).to(torch.bfloat16)


class Batch:
    """Requests (rows, keys) over shuffled pages; what no request holds is NaN, table entries past a request's end are far outside."""

    def __init__(self, reqs, Hq, Hkv, D, page, seed=1, extra_width=1, behind=3):
        self.reqs, self.Hq, self.Hkv, self.D, self.page = reqs, Hq, Hkv, D, page
        need = [-(-n // page) for _, n in reqs]
        n_pages, width = sum(need) + 2, max(need) + extra_width
        g = gen(seed)
        order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        k, v = (torch.full((n_pages, Hkv, page, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        table = torch.full((len(reqs), width), 1 << 30, dtype=torch.int32, device=DEV)
        table[:, ::2] = -7
        used = 0
        for b, (r, n) in enumerate(reqs):
            table[b, :need[b]] = order[used:used + need[b]]
            used += need[b]
            j = torch.arange(n, device=DEV)
            for c in (k, v):
                c[table[b, j // page].long(), :, j % page] = torch.randn(n, Hkv, D, generator=g, device=DEV).to(torch.bfloat16)
        self.cache, self.table = gmlp.KvCache(k, v), table
        self.lengths = torch.tensor([n for _, n in reqs], dtype=torch.int32, device=DEV)
        start = [0]
        for r, _ in reqs:
            start.append(start[-1] + r)
        self.rows = start[-1]
        self.start = torch.tensor(start, dtype=torch.int32, device=DEV)
        self.Q = torch.randn(self.rows + behind, Hq * D, generator=g, device=DEV).to(torch.bfloat16)

    def run(self, **kw):
        O = torch.full_like(self.Q, 7.0)
        return gmlp.kv_attention(self.Q, self.cache, self.table, self.lengths, self.Hq, q_start=self.start, O=O, checked=True, **kw)

    def keys(self, b):
        return (P.rows_of(c, self.table[b], self.reqs[b][1]) for c in (self.cache.k, self.cache.v))

    def check(self, scale=None, causal=True, only=None):
        O = self.run(scale=scale, causal=causal)
        assert bool((O[self.rows:] == 7.0).all())                        # rows of no request
        self.check_rows(O, scale, causal, only)
        return O

    def check_rows(self, O, scale=None, causal=True, only=None):
        at = 0
        for b, (r, n) in enumerate(self.reqs):
            if only is None or b in only:
                k, v = self.keys(b)
                want, A, E = P.attention(self.Q[at:at + r], k, v, self.Hq, self.D ** -0.5 if scale is None else scale, causal)
                if r:
                    worst = float(((O[at:at + r].double() - want).abs() / P.attention_bound(want, A, E, self.D, n)).nan_to_num(nan=math.inf).max())
                    assert worst <= 1.0, (b, r, n, worst)
            at += r


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 385, 1000, 4097])
def test_single_tokens(n, D):
    Batch([(1, n)], 8, 2, D, 16, seed=n).check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("r", [2, 3, 15, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 300, 511])
def test_chunks(r, D):
    Batch([(r, 700)], 8, 2, D, 64, seed=r).check()


@pytest.mark.parametrize("r", [1, 2, 17, 64, 128, 129, 1000])
def test_whole_prompts(r):
    Batch([(r, r)], 4, 2, 128, 32, seed=r).check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (6, 2), (12, 4), (10, 2), (7, 1), (24, 2), (16, 1), (50, 1), (64, 1), (65, 1), (100, 1), (128, 1)])
@pytest.mark.parametrize("r", [1, 5, 150])
def test_head_layouts(Hq, Hkv, D, r):
    Batch([(r, 333)], Hq, Hkv, D, 16, seed=Hq).check()


@pytest.mark.parametrize("page", [16, 32, 48, 64, 80, 96, 112, 128, 192, 256, 1024])
@pytest.mark.parametrize("r", [1, 90])
def test_page_sizes(page, r):
    Batch([(r, 777), (1, page), (r, page + 90)], 8, 2, 128, page, seed=page).check()
    Batch([(r, 1153)], 4, 2, 64, page, seed=page).check()


RAGGED = [(1, 300), (1, 1), (200, 200), (0, 50), (3, 0), (1, 2000), (77, 500), (5, 2), (0, 0), (1, 129), (130, 129), (16, 1024)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,Hkv,D,page", [(8, 2, 128, 64), (12, 4, 64, 48), (16, 2, 128, 16), (6, 6, 64, 128)])
def test_ragged_batches(Hq, Hkv, D, page, causal):
    Batch(RAGGED, Hq, Hkv, D, page).check(causal=causal)


def test_many_requests():
    reqs = [(1 + (b % 7 == 0) * 30, 31 + (b * 37) % 400) for b in range(700)]
    Batch(reqs, 8, 2, 64, 32).check(only=range(0, 700, 23))


def test_thousands_of_empty_places():
    """A padded batch of many places, most of them without a key, some without a row."""
    reqs = [(b % 2, 0) for b in range(20000)]
    reqs[17], reqs[9000], reqs[19999] = (1, 100), (40, 200), (1, 7)
    batch = Batch(reqs, 4, 1, 64, 16)
    O = batch.check(only=(17, 9000, 19999))
    at = int(batch.start[9001])
    assert bool((O[18:int(batch.start[9000])] == 0).all()) and bool((O[at:batch.rows - 1] == 0).all())


@pytest.mark.parametrize("reqs,Hq,Hkv,D,page", [([(1, 70000)], 64, 8, 128, 64), ([(61, 30000)], 16, 2, 128, 64), ([(300, 20000)], 8, 1, 64, 128),
                                                ([(1, 40000), (1, 50), (600, 3000), (1, 9000)], 16, 4, 128, 16), ([(2, 131071)], 4, 1, 64, 48)])
def test_long(reqs, Hq, Hkv, D, page):
    Batch(reqs, Hq, Hkv, D, page).check()


@pytest.mark.parametrize("reqs,Hq,Hkv,D,page", [([(1, 300), (2000, 2100), (1, 5000), (3, 40)], 8, 2, 128, 64),       # single tokens beside a long chunk
                                                ([(1500, 3000)], 32, 8, 128, 64), ([(1200, 1200), (1300, 4000)], 12, 4, 64, 48),
                                                ([(33, 6000)] * 12, 8, 2, 128, 32), ([(20, 3000)] * 9, 16, 4, 64, 16),  # every cut item has one tile
                                                ([(1, 700)] * 300, 8, 2, 128, 64), ([(4, 1100)] * 90, 8, 2, 64, 16)])
def test_items_of_each_kind_cut_between_ctas(reqs, Hq, Hkv, D, page):
    Batch(reqs, Hq, Hkv, D, page).check(only=range(0, len(reqs), max(1, len(reqs) // 12)))


@pytest.mark.parametrize("n", [300, 1400, 1401, 1535, 1536, 1537, 1700])
@pytest.mark.parametrize("r", [1, 20, 40])
def test_around_the_length_that_is_cut(n, r):
    Batch([(r, n)] * 40, 8, 2, 128, 64).check(only=range(0, 40, 7))


@pytest.mark.parametrize("B,n,r", [(18, 1000, 1), (16, 1500, 1), (16, 4000, 1), (17, 4000, 1), (40, 700, 1), (16, 2000, 20), (9, 900, 60)])
@pytest.mark.parametrize("spread", [0, 1, 100, 400])
def test_batches_of_nearly_the_same_length(B, n, r, spread):
    """Whether such items are cut depends on their number and on the shortest and the longest of them."""
    Batch([(r, n - spread * (b % 3) // 2) for b in range(B)] + [(0, 50)], 32, 8, 128, 64).check()


def test_wide_tables_and_uniform_rows():
    batch = Batch([(4, 100), (4, 3), (4, 1500)], 8, 2, 128, 64, extra_width=5000, behind=0)
    O = batch.check()
    same = gmlp.kv_attention(batch.Q, batch.cache, batch.table, batch.lengths, 8, q_len=4, checked=True)
    assert torch.equal(O, same)


@pytest.mark.parametrize("scale", [1e-6, 0.7, 3.0])
def test_scales(scale):
    Batch([(1, 500), (150, 400)], 8, 2, 128, 64).check(scale=scale)


@pytest.mark.parametrize("r", [1, 200])
@pytest.mark.parametrize("slope", [0.05, 2.0, -2.0, 40.0, -40.0])
def test_scores_that_rise_or_fall_along_the_keys(slope, r):
    """The running base of the exponentials has to move a little, by hundreds or by thousands of binary orders, or stay."""
    batch = Batch([(r, 900)], 8, 2, 128, 64)
    u = torch.randn(128, generator=gen(3), device=DEV)
    u = 4 * u / u.norm()
    j = torch.arange(900, device=DEV)
    batch.cache.k[batch.table[0, j // 64].long(), :, j % 64] = ((1 + slope * j)[:, None, None] * u).expand(900, 2, 128).to(torch.bfloat16)
    batch.Q[:] = ((1 + torch.rand(batch.Q.shape[0], 1, generator=gen(4), device=DEV)) * u.repeat(8)).to(torch.bfloat16)
    batch.check()


def test_scores_far_below_zero():
    """Every score is some -10^6: the base is far from zero, in every part of the keys."""
    batch = Batch([(1, 3000), (200, 700)], 4, 1, 64, 64)
    batch.Q[:, ::64], batch.cache.k[..., 0] = 1e3, torch.where(torch.isnan(batch.cache.k[..., 0]), batch.cache.k[..., 0], -8192.0)
    batch.check()


def test_one_key_is_that_value():
    batch = Batch([(1, 1), (1, 1)], 8, 2, 128, 16)
    O = batch.check()
    for b in range(2):
        _, v = batch.keys(b)
        assert torch.equal(O[b].view(8, 128), v[0].repeat_interleave(4, 0))


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 4, 64), (7, 1, 128)])
@pytest.mark.parametrize("r,n", [(5, 300), (100, 300), (300, 300), (150, 130), (16, 4000)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_hidden_rows_that_are_no_numbers_stay_hidden(r, n, value, Hq, Hkv, D):
    """The newest key and value hold `value` in some channels: earlier positions do not see them; the last one does."""
    batch = Batch([(r, n), (1, 50)], Hq, Hkv, D, 32)
    clean = batch.run().clone()
    last = (batch.table[0, (n - 1) // 32].long(), 0, (n - 1) % 32)
    batch.cache.v[last][3], batch.cache.v[last][D - 1] = value, value
    O = batch.run()
    ratio = Hq // Hkv
    hit = torch.zeros(O.shape[0], Hq, D, dtype=torch.bool, device=DEV)
    hit[r - 1, :ratio, [3, D - 1]] = True
    o = O.view(-1, Hq, D)
    assert bool(torch.isnan(o[hit]).all()) if math.isnan(value) else bool((o[hit] == value).all())
    assert torch.equal(o[~hit], clean.view(-1, Hq, D)[~hit])
    batch.cache.k[last][5] = value                                       # a key that is no number: its row of scores
    o = batch.run().view(-1, Hq, D)
    rows = torch.ones(O.shape[0], Hq, dtype=torch.bool, device=DEV)
    rows[r - 1, :ratio] = False
    assert torch.equal(o[rows], clean.view(-1, Hq, D)[rows])


def test_queries_that_are_no_numbers_stay_in_their_row_and_head():
    batch = Batch([(90, 300), (1, 70)], 8, 2, 128, 64)
    clean = batch.run().clone()
    batch.Q[7, 130], batch.Q[90, 5] = float("nan"), float("nan")
    o, c = batch.run().view(-1, 8, 128), clean.view(-1, 8, 128)
    hit = torch.zeros(o.shape[:2], dtype=torch.bool, device=DEV)
    hit[7, 1], hit[90, 0] = True, True
    assert bool(torch.isnan(o[hit]).all()) and torch.equal(o[~hit], c[~hit])


def test_infinite_scores():
    """A key that scores -infinity has no weight; a row whose scores are all -infinity gets zeros."""
    batch = Batch([(1, 200), (1, 30), (150, 200)], 2, 1, 64, 16, behind=0)
    batch.Q[:, 0], batch.Q[:, 64] = 2.0, 2.0
    for b, some in ((0, [3, 150]), (1, list(range(30))), (2, [0, 60, 199])):
        for j in some:
            batch.cache.k[batch.table[b, j // 16].long(), 0, j % 16, 0] = -float("inf")
    O = batch.run()
    assert bool((O[1] == 0).all()) and bool(torch.isfinite(O).all())
    at = 0
    for b, (r, n) in enumerate(batch.reqs):
        k, v = batch.keys(b)
        ok = torch.isfinite(k).all(-1)[:, 0]
        q = batch.Q[at:at + r].double().view(r, 2, 64)
        s = torch.einsum("rhd,nd->rhn", q, torch.where(ok[:, None], k[:, 0].double(), 0.0)) / 8
        seen = ok & (torch.arange(n, device=DEV) <= torch.arange(r, device=DEV)[:, None] + n - r)
        p = torch.where(seen[:, None], s, -math.inf).softmax(-1).nan_to_num(0.0)
        want = torch.einsum("rhn,nd->rhd", p, v[:, 0].double()).reshape(r, -1)
        A = torch.einsum("rhn,nd->rhd", p, v[:, 0].double().abs()).reshape(r, -1)
        E = (torch.einsum("rhd,nd->rhn", q.abs(), torch.where(ok[:, None], k[:, 0].double().abs(), 0.0)) / 8).amax(-1, keepdim=True).expand(r, 2, 64).reshape(r, -1)
        assert bool(((O[at:at + r].double() - want).abs() <= P.attention_bound(want, A, E, 64, n)).all())
        at += r


def test_bad_pages_lengths_and_starts_are_left_out_and_reported():
    reqs = [(1, 300), (90, 400), (1, 70), (2, 40)]
    batch = Batch(reqs, 8, 2, 64, 16, behind=0)
    holes = {0: [3], 1: [0, 7, 24]}
    for b, pages in holes.items():
        for i, p in enumerate(pages):
            batch.table[b, p] = (-1, 1 << 30, batch.cache.n_pages)[i]
    with pytest.raises(gmlp.GmlpError) as e:
        batch.run()
    assert e.value.status == gmlp.ERR_INDEX and gmlp.device_status() == 0
    O = torch.full_like(batch.Q, 7.0)
    gmlp.kv_attention(batch.Q, batch.cache, batch.table, batch.lengths, 8, q_start=batch.start, O=O)
    assert gmlp.device_status() >> 16 == 200
    batch.check_rows(O, only=(2, 3))
    at = 0
    for b, pages in holes.items():                                       # the other keys, each with its own place in the mask
        r, n = reqs[b]
        ok = torch.tensor([j // 16 not in pages for j in range(n)], device=DEV)
        t = batch.table[b].clone()
        t[pages] = 0
        k, v = (P.rows_of(c, t, n)[ok].double() for c in (batch.cache.k, batch.cache.v))
        seen = (torch.arange(n, device=DEV) <= torch.arange(r, device=DEV)[:, None] + n - r)[:, ok]
        q = batch.Q[at:at + r].double().view(r, 2, 4, 64)
        s = torch.where(seen[:, None, None], torch.einsum("rghd,ngd->rghn", q, k) / 8, -math.inf)
        p = s.softmax(-1).nan_to_num(0.0)
        want, A = (torch.einsum("rghn,ngd->rghd", p, x).reshape(r, -1) for x in (v, v.abs()))
        E = torch.full_like(want, float((q.abs().sum(-1).max() * k.abs().max()) / 8))
        assert bool(((O[at:at + r].double() - want).abs() <= P.attention_bound(want, A, E, 64, n)).all())
        at += r
    batch = Batch(reqs, 8, 2, 64, 16, behind=0)
    for bad in (-5, 16 * batch.table.shape[1] + 1, (1 << 31) - 1):       # a bad length: that request's keys are left out
        batch.lengths[1] = bad
        O = torch.full_like(batch.Q, 7.0)
        gmlp.kv_attention(batch.Q, batch.cache, batch.table, batch.lengths, 8, q_start=batch.start, O=O)
        assert gmlp.device_status() >> 16 == 200
        assert bool((O[1:91] == 0).all())
        batch.check_rows(O, only=(0, 2, 3))                              # (they may be split elsewhere than beside a good length)
    batch.lengths[1] = 400
    for i, bad in ((1, -3), (1, 1 << 30), (2, 95)):                      # starts that fall or pass the rows: those requests' rows are left out
        start = batch.start.clone()
        start[i] = bad
        O = torch.full_like(batch.Q, 7.0)
        gmlp.kv_attention(batch.Q, batch.cache, batch.table, batch.lengths, 8, q_start=start, O=O)
        assert gmlp.device_status() >> 16 == 200
        s = start.tolist()
        for b in range(4):
            if not 0 <= s[b] <= s[b + 1] <= batch.Q.shape[0]:
                covered = any(0 <= s[c] <= int(batch.start[b]) < s[c + 1] <= batch.Q.shape[0] for c in range(4))
                assert covered or bool((O[batch.start[b]:batch.start[b + 1]] == 7.0).all())
            elif (s[b], s[b + 1]) == (int(batch.start[b]), int(batch.start[b + 1])):
                batch.check_rows(O, only=(b,))


def test_cache_past_four_gigabytes():
    n_pages, page, Hkv, D = 36000, 64, 8, 128
    k, v = (torch.empty(n_pages, Hkv, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    border = (1 << 32) // (Hkv * page * D * 2)
    pages = torch.tensor([n_pages - 1, border - 1, border, 0, n_pages - 2, border + 1], device=DEV)
    n = 64 * 6 - 5
    k[pages], v[pages] = bf16(1, 6, Hkv, page, D), bf16(2, 6, Hkv, page, D)
    table = pages.to(torch.int32)[None]
    for r in (1, 100):
        Q = bf16(3, r, 32 * D)
        O = gmlp.kv_attention(Q, gmlp.KvCache(k, v), table, torch.tensor([n], dtype=torch.int32, device=DEV), 32, q_len=r, checked=True)
        want, A, E = P.attention(Q, P.rows_of(k, table[0], n), P.rows_of(v, table[0], n), 32, D ** -0.5)
        assert bool(((O.double() - want).abs() <= P.attention_bound(want, A, E, D, n)).all())


@pytest.mark.parametrize("reqs", [[(1, 4000)] * 3, [(500, 2000), (1, 700)]])
def test_repeats_bit_for_bit_on_streams_and_in_graphs(reqs):
    batch = Batch(reqs, 8, 2, 128, 64)
    want = batch.run().clone()
    side, call = torch.cuda.Stream(), lambda **kw: gmlp.kv_attention(batch.Q, batch.cache, batch.table, batch.lengths, 8, q_start=batch.start, **kw)
    side.wait_stream(torch.cuda.current_stream())
    outs = [call(stream=s)[:batch.rows] for s in (side, None) for _ in range(3)]        # two calls at once
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[:batch.rows]) for o in outs)
    ws = torch.empty(max(256, gmlp.kv_workspace_bytes(batch.Q.shape[0], 8, 2, 128)), dtype=torch.uint8, device=DEV)
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:                                                                    # two captured calls that share a workspace
        with torch.cuda.graph(g):
            outs.append(call(workspace=ws))
    lengths = batch.lengths.clone()
    for i in range(4):
        ws.fill_(i * 85)                                                                # no state is kept in it
        batch.lengths.copy_(lengths - 100 * (i % 2))
        graphs[i % 2].replay()
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0][:batch.rows], outs[1][:batch.rows])
        assert torch.equal(outs[0][:batch.rows], want[:batch.rows]) == (i % 2 == 0)
    batch.lengths.copy_(lengths)
    del graphs


@pytest.mark.parametrize("reqs,most", [([(1, 3000)] * 16, 1.05), ([(16, 2000)] * 4, 1.05), ([(300, 1500)] * 2, 1.5), ([(1, 131071)], 1.05)])
def test_accuracy_by_the_error_s_norm(reqs, most):
    """The error's norm over that of the last rounding alone: two bf16 terms of a probability add next to nothing; one term, in tiles of
    more than 128 rows, an error of the same size as the last rounding's: a square root of two."""
    batch = Batch(reqs, 8, 2, 128, 64, behind=0)
    O = batch.run()
    at, err, own = 0, 0.0, 0.0
    for b, (r, n) in enumerate(batch.reqs):
        want, _, _ = P.attention(batch.Q[at:at + r], *batch.keys(b), 8, 128 ** -0.5)
        err += float((O[at:at + r].double() - want).square().sum())
        own += float((want.to(torch.bfloat16).double() - want).square().sum())
        at += r
    assert (err / own) ** 0.5 <= most, (err / own) ** 0.5


def test_the_most_requests_and_rows():
    """65535 requests (places of a padded batch among them) that share their pages, and 2^24 rows of one request."""
    g, D = gen(1), 64
    k, v = (torch.randn(5, 1, 16, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    cache, B = gmlp.KvCache(k, v), 65535
    lengths = torch.randint(0, 40, (B,), generator=g, device=DEV).to(torch.int32)
    table = torch.randint(0, 5, (B, 3), generator=g, device=DEV).to(torch.int32)
    Q = torch.randn(B, D, generator=g, device=DEV).to(torch.bfloat16)
    O = gmlp.kv_attention(Q, cache, table, lengths, 1, checked=True)
    j = torch.arange(48, device=DEV)
    for lo in range(0, B, 8192):
        rows = slice(lo, min(B, lo + 8192))
        kk, vv = (c[table[rows].long(), 0].flatten(1, 2).double() for c in (k, v))
        s = torch.einsum("bd,bnd->bn", Q[rows].double(), kk) / 8
        p = torch.where(j < lengths[rows, None], s, -math.inf).softmax(-1).nan_to_num(0.0)
        want, A = torch.einsum("bn,bnd->bd", p, vv), torch.einsum("bn,bnd->bd", p, vv.abs())
        E = (torch.einsum("bd,bnd->bn", Q[rows].double().abs(), kk.abs()) / 8).amax(-1, keepdim=True).expand_as(want)
        assert bool(((O[rows].double() - want).abs() <= P.attention_bound(want, A, E, D, 48)).all())
    T = 1 << 24
    Q = torch.randn(T, D, generator=g, device=DEV, dtype=torch.bfloat16)
    n = torch.tensor([70], dtype=torch.int32, device=DEV)
    table = torch.arange(5, dtype=torch.int32, device=DEV)[None]
    O = gmlp.kv_attention(Q, cache, table, n, 1, q_len=T, checked=True)
    assert int(torch.count_nonzero(O[:T - 70])) == 0
    kk, vv = (P.rows_of(c, table[0], 70) for c in (k, v))
    want, A, E = P.attention(Q[T - 200:], kk, vv, 1, 0.125)
    assert bool(((O[T - 200:].double() - want).abs() <= P.attention_bound(want, A, E, D, 70)).all())
    O = gmlp.kv_attention(Q, cache, table, n, 1, q_len=T, causal=False, checked=True)
    for at in (0, 255, 256, T // 2, T - 200):
        want, A, E = P.attention(Q[at:at + 200], kk, vv, 1, 0.125, causal=False)
        assert bool(((O[at:at + 200].double() - want).abs() <= P.attention_bound(want, A, E, D, 70)).all())


def test_workspaces_of_the_caller():
    batch = Batch([(3, 2000), (200, 300)], 8, 2, 64, 16, behind=0)
    want, need = batch.run().clone(), gmlp.kv_workspace_bytes(batch.Q.shape[0], 8, 2, 64)
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(batch.run(workspace=ws[:need]), want)
    assert bool((ws[need:] == 255).all())                                # nothing behind it is touched
    for bad, status in ((ws[:need - 1], gmlp.ERR_WORKSPACE), (ws[16:], gmlp.ERR_ALIGN)):
        with pytest.raises(gmlp.GmlpError) as e:
            batch.run(workspace=bad)
        assert e.value.status == status
    with pytest.raises(ValueError):
        batch.run(workspace=torch.empty(need, dtype=torch.uint8))


def test_refusals_of_the_binding():
    batch = Batch([(2, 40), (3, 20)], 8, 2, 64, 16, behind=0)
    ok = dict(Q=batch.Q, cache=batch.cache, block_table=batch.table, lengths=batch.lengths, n_q_heads=8, q_start=batch.start)
    for bad in (dict(Q=batch.Q.float()), dict(block_table=batch.table.long()), dict(lengths=batch.lengths.cpu()), dict(q_start=batch.start.long()),
                dict(O=batch.Q.float())):
        with pytest.raises(TypeError):
            gmlp.kv_attention(**{**ok, **bad})
    for bad in (dict(n_q_heads=4), dict(q_start=batch.start[:-1]), dict(q_start=None), dict(lengths=batch.lengths[:1]), dict(block_table=batch.table[0]),
                dict(O=batch.Q[:2])):
        with pytest.raises(ValueError):
            gmlp.kv_attention(**{**ok, **bad})
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.kv_attention(**{**ok, "scale": 0.0})
    assert e.value.status == gmlp.ERR_FLAGS
    empty = gmlp.kv_attention(batch.Q[:0], batch.cache, batch.table[:0], batch.lengths[:0], 8, q_start=batch.start[:1])
    assert empty.shape == (0, 512)
