"""The paged cache's calls against their plain forms in 64 bits (tests/paged_ref.py, which derives the bounds)."""
import math

import pytest
import torch

import paged_ref as R
from paper_2605_18753_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


class Setup:
    """A cache on the GPU and its copy on the CPU.  layout "token": pages [n_pages, page, h_kv, d] seen as
    [n_pages, h_kv, page, d]; slack: elements between heads that no call may touch."""

    def __init__(self, lens, news, h_kv=2, g=4, d=128, page=16, dtype=BF, seed=0, spare=0, behind=0.0, layout="head", qscale=1.0, width=None):
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
        B_ = len(lens)
        per = [-(-n // page) for n in lens]
        n_pages = sum(per) + 2
        ids = torch.randperm(n_pages, generator=gen)[:sum(per)].tolist()
        width = width or max(max(per), 1)
        table = torch.full((B_, width), -1, dtype=torch.int32)
        at = 0
        for b, k in enumerate(per):
            table[b, :k] = torch.tensor(ids[at:at + k], dtype=torch.int32)
            at += k
        shape = (n_pages, h_kv, page, d)
        k, v = rand(*shape).to(dtype), rand(*shape).to(dtype)
        if behind:                                              # what the pages hold behind the sequences' ends
            used = torch.zeros((n_pages, page), dtype=torch.bool)
            for b, n in enumerate(lens):
                i = torch.arange(n)
                used[table[b].long()[i // page], i % page] = True
            k = torch.where(used[:, None, :, None], k, torch.tensor(behind).to(dtype))
            v = torch.where(used[:, None, :, None], v, torch.tensor(behind).to(dtype))
        start = [0]
        for m in news:
            start.append(start[-1] + m)
        self.row_start = torch.tensor(start, dtype=torch.int32)
        self.rows = start[-1] + spare
        self.q = (qscale * rand(max(self.rows, 1), h_kv * g, d)).to(dtype)
        self.h_kv, self.g = h_kv, g
        lens_t = torch.tensor(lens, dtype=torch.int32)
        self.ref = R.Cache(k, v, table, lens_t)
        kg, vg = k.to(DEV), v.to(DEV)
        if layout == "token":
            kg, vg = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kg, vg))
        self.gpu = B.PagedCache(kg, vg, table.to(DEV), lens_t.to(DEV))
        self.start_gpu = self.row_start.to(DEV)

    def params(self, causal=True, scale=0.0):
        return B.make_paged_params(self.gpu, self.q.shape[0], self.h_kv * self.g, causal=causal, scale=scale)

    def attend(self, causal=True, scale=0.0, q=None, stream=None):
        p = self.params(causal, scale)
        q = self.q.to(DEV) if q is None else q
        o = torch.full((q.shape[0], q.shape[1], q.shape[2]), 77.0, dtype=q.dtype, device=DEV)
        lse = torch.full(q.shape[:2], 77.0, dtype=F32, device=DEV)
        ws = B.alloc_paged_workspace(p, DEV)
        ws.fill_(255)                                           # NaN everywhere
        B.dash_paged_attend(p, self.gpu, q, self.start_gpu, o, ws, lse=lse)
        torch.cuda.synchronize()
        return o.cpu(), lse.cpu()

    def check_attend(self, causal=True, scale=0.0):
        o, lse = self.attend(causal, scale)
        want, wl, tol, ltol = R.attend(self.ref, self.q, self.row_start, self.h_kv, causal, scale or None)
        own = int(self.row_start[-1])
        assert (o[own:].float() == 77).all() and (lse[own:] == 77).all()          # rows of no sequence
        o, lse, want, wl, tol, ltol = (x[:own] for x in (o, lse, want, wl, tol, ltol))
        assert torch.equal(torch.isneginf(lse), torch.isneginf(wl))
        seen = ~torch.isneginf(wl)
        assert ((lse.double() - wl).abs()[seen] <= ltol[seen]).all(), float(((lse.double() - wl).abs() / ltol)[seen].max())
        bad = (o.double() - want).abs() / tol.clamp(min=1e-30)
        assert not torch.isnan(o).any()
        assert ((o.double() - want).abs() <= tol).all(), float(bad.max())
        return lse


EDGE = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_single_tokens_at_the_edges_of_tiles_and_pages(dtype, d, page):
    s = Setup(EDGE, [1] * len(EDGE), d=d, page=page, dtype=dtype, behind=math.nan, seed=1)
    s.check_attend()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h_kv,g", [(1, 1), (3, 2), (2, 8), (1, 16), (8, 4), (5, 1)])
def test_head_layouts(dtype, h_kv, g):
    s = Setup([300, 41, 1000], [1, 3, 20], h_kv=h_kv, g=g, dtype=dtype, page=32, seed=2)
    s.check_attend()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("news", [[7, 0, 33, 1, 130, 64], [1, 1, 0, 0, 0, 1], [0, 0, 0, 0, 700, 0]])
def test_chunks_of_every_length_beside_each_other(dtype, causal, news):
    s = Setup([500, 20, 33, 1, max(131, news[4]), 64], news, dtype=dtype, page=16, spare=3, behind=math.inf, seed=3)
    s.check_attend(causal)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_whole_prompts(dtype, d):
    s = Setup([257, 100, 513], [257, 100, 513], h_kv=2, g=2, d=d, dtype=dtype, page=64, behind=math.nan, seed=4)
    s.check_attend()


# tables wide enough for tiles of 128 rows, whatever the lengths
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,page,h_kv,g", [(128, 16, 2, 4), (64, 16, 3, 2), (128, 64, 1, 16), (64, 256, 2, 8), (128, 32, 4, 1)])
@pytest.mark.parametrize("news", [[7, 0, 33, 1, 130, 64, 9], [40, 20, 0, 1, 0, 3, 0], [0, 0, 0, 0, 700, 0, 0]])
def test_chunks_in_wide_tables(causal, d, page, h_kv, g, news):
    s = Setup([500, 20, 33, 1, max(131, news[4]), 64, 0], news, h_kv=h_kv, g=g, d=d, page=page, spare=3, behind=math.inf, seed=36, width=4096 // page)
    s.check_attend(causal)


@pytest.mark.parametrize("lens,news", [([6400], [380]), ([6300], [600]), ([6400, 70, 6000], [250, 1, 129])])
def test_items_that_stay_whole_beside_cut_ones(lens, news):
    Setup(lens, news, h_kv=128, g=1, d=64, page=128, seed=41).check_attend()


# A workgroup that walks more than 64 pages asks for the next 64 entries of the table on the way.  Whole items of 400 and 200 pages beside parts of 136 and 68;
# parts of 24 and of 46 tiles, 96 and 184 pages of 16, most of which begin inside the sequence.
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,news,h_kv,g,d,page", [([6400], [380], 128, 1, 64, 16), ([6400], [380], 128, 1, 64, 32), ([9000, 70], [300, 1], 8, 4, 128, 16),
                                                     ([17600, 40], [20, 5], 64, 8, 64, 16)])
def test_items_of_many_pages(lens, news, h_kv, g, d, page, causal):
    Setup(lens, news, h_kv=h_kv, g=g, d=d, page=page, behind=math.inf, seed=44).check_attend(causal)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h_kv,g,d,longest,causal", [(8, 4, 64, 900, True), (8, 2, 128, 1500, False), (16, 1, 64, 3000, True)])
def test_single_tokens_in_wide_tables(dtype, h_kv, g, d, longest, causal):
    lens = [longest if i == 11 else (61 * i) % 900 for i in range(32)]
    s = Setup(lens, [min(1 + i % 2, 2) for i in range(32)], h_kv=h_kv, g=g, d=d, page=64, dtype=dtype, behind=math.nan, seed=40, width=128)
    s.check_attend(causal)


@pytest.mark.parametrize("h_kv,g,d,batch,new", [(8, 1, 64, 30, 130), (16, 4, 128, 14, 30), (8, 2, 64, 70, 20), (32, 1, 64, 6, 140)])
def test_items_of_unequal_lengths_are_cut_finely(h_kv, g, d, batch, new):
    lens = [max(new, 2600 if i % 7 == 3 else (97 * i) % 200) for i in range(batch)]
    Setup(lens, [new] * batch, h_kv=h_kv, g=g, d=d, page=64, seed=39).check_attend()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 128])
def test_whole_prompts_in_wide_tables(d, page):
    s = Setup(EDGE, EDGE, h_kv=2, g=4, d=d, page=page, behind=math.nan, seed=37, width=4096 // page)
    s.check_attend()
    s = Setup([5, 0, 20, 1], [90, 64, 300, 33], d=d, page=page, behind=math.nan, seed=38, width=4096 // page)
    lse = s.check_attend()
    assert torch.isneginf(lse).sum() == (85 + 64 + 280 + 32) * 8


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_that_see_nothing(dtype):
    # more new tokens than the cache holds: the first of them lie before slot 0
    s = Setup([5, 0, 20], [9, 4, 30], dtype=dtype, behind=math.nan, seed=5)
    lse = s.check_attend()
    assert torch.isneginf(lse).sum() == (4 + 4 + 10) * 8


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,news", [(5000, 1), (5000, 40), (20001, 2), (9000, 300)])
def test_long_caches_are_cut_and_joined(dtype, n, news):
    s = Setup([n, 70], [news, 1], h_kv=1, g=4, dtype=dtype, page=64, seed=6)
    s.check_attend()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h_kv,g,lens,news", [(1, 16, [17000, 30], [1, 1]), (1, 8, [8200, 9000, 50], [2, 1, 0]), (2, 16, [4100], [1]), (1, 1, [40000], [3]),
                                              (4, 4, [2177], [4])])
@pytest.mark.parametrize("d", [64, 128])
def test_long_caches_of_few_heads_are_joined_in_levels(dtype, h_kv, g, lens, news, d):
    Setup(lens, news, h_kv=h_kv, g=g, d=d, dtype=dtype, page=64, seed=34).check_attend()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_join_in_levels_in_a_captured_graph(dtype):
    s = Setup([17000], [1], h_kv=1, g=16, d=64, dtype=dtype, page=64, seed=35)
    p, q = s.params(), s.q.to(DEV)
    o, lse, ws = torch.empty_like(q), torch.empty((1, 16), device=DEV), B.alloc_paged_workspace(p, DEV)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        B.dash_paged_attend(p, s.gpu, q, s.start_gpu, o, ws, lse=lse)
    for n in (17000, 900, 16500, 8191, 3, 17000):               # as many pieces as there are runs, some, one
        s.gpu.lens[0] = n
        s.ref.lens[0] = n
        want, wl = s.attend()
        for _ in range(3):
            o.fill_(77.0)
            lse.fill_(77.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o.cpu(), want) and torch.equal(lse.cpu(), wl)


def test_peaked_and_falling_logits():
    # logits of several hundred in rising and in falling order: the running maximum moves all the way, or never
    for sign in (1.0, -1.0):
        s = Setup([700], [3], h_kv=1, g=1, page=16, seed=7)
        ramp = torch.linspace(-3, 3, 700) * sign
        s.ref.k.zero_()
        page, off = s.ref.where(0, 700)
        s.ref.k[page, 0, off, 0] = ramp.to(BF)
        s.q.zero_()
        s.q[:, 0, 0] = 1000.0
        s.gpu.k.copy_(s.ref.k)
        s.check_attend()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strided_queries_outputs_and_pages(dtype):
    check_strides(Setup([100, 333], [5, 80], dtype=dtype, page=32, layout="token", seed=8), dtype)
    check_strides(Setup([100, 333], [5, 80], dtype=dtype, page=32, layout="token", seed=8, width=64), dtype)


def check_strides(s, dtype):
    s.check_attend()
    big = torch.full((s.rows, 2 * 8, 128 + 8), 5.0, dtype=dtype, device=DEV)
    q = big[:, 8:, 8:]
    q.copy_(s.q)
    o, _ = s.attend(q=q)
    plain, _ = s.attend()
    assert torch.equal(o, plain)
    p = s.params()
    out = torch.full((8, s.rows, 128 + 64), 3.0, dtype=dtype, device=DEV)
    view = out[:, :, :128].transpose(0, 1)
    B.dash_paged_attend(p, s.gpu, s.q.to(DEV), s.start_gpu, view, B.alloc_paged_workspace(p, DEV))
    assert torch.equal(view.cpu(), plain) and (out[:, :, 128:] == 3).all()


def test_a_batch_of_more_sequences_than_a_wave_has_lanes():
    lens = [(37 * i) % 400 for i in range(150)]
    s = Setup(lens, [min(1 + (i % 3 == 0), 2) if i % 7 else 0 for i in range(150)], h_kv=1, g=2, d=64, page=16, seed=9)
    s.check_attend()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_chunks_of_more_sequences_than_a_wave_has_lanes(dtype):
    lens = [(53 * i) % 300 + 30 for i in range(100)]
    s = Setup(lens, [(7 * i) % 30 if i % 5 else 0 for i in range(100)], h_kv=1, g=4, d=64, page=16, dtype=dtype, seed=32)
    s.check_attend()
    check_weigh(s)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page,d", [(512, 128), (1024, 64)])
def test_large_pages(dtype, page, d):
    for news in ([1, 1, 1, 1], [3, 70, 600, 0]):
        s = Setup([page, 2 * page + 1, 1500, page - 1], news, d=d, page=page, dtype=dtype, behind=math.nan, seed=45)
        s.check_attend()
        check_weigh(s)
    gen = torch.Generator().manual_seed(46)
    pos, seen = positions(s, gen)
    s = Setup([page, 2 * page + 1, 1500, page - 1], [1] * 4, d=d, page=page, g=1, dtype=dtype, seed=45)
    evict_both(s, 700, 4, 30, torch.randn(s.ref.k.shape[:3], generator=gen).exp(), pos, seen)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("news,width", [([2, 1, 0], None), ([40, 17, 3], 128), ([100, 1, 2], 128)])
def test_rows_before_the_first_sequence(dtype, news, width):
    s = Setup([300, 41, 90], news, h_kv=2, g=4, dtype=dtype, page=32, spare=5, seed=47, width=width)
    s.row_start += 5
    s.start_gpu = s.row_start.to(DEV)
    o, lse = s.attend()
    want, wl, tol, ltol = R.attend(s.ref, s.q, s.row_start, 2)
    assert (o[:5].float() == 77).all() and (lse[:5] == 77).all()
    assert ((o[5:].double() - want[5:]).abs() <= tol[5:]).all() and ((lse[5:].double() - wl[5:]).abs() <= ltol[5:]).all()
    lse[:5] = math.nan
    s.q[:5] = math.nan
    check_weigh(s, lse=lse)
    new = torch.randn((2, s.rows, 2, 128)).to(dtype)
    B.dash_paged_append(s.params(), s.gpu, new[0].to(DEV), new[1].to(DEV), s.start_gpu)
    R.append(s.ref, new[0], new[1], s.row_start)
    assert torch.equal(s.gpu.k.cpu(), s.ref.k) and torch.equal(s.gpu.v.cpu(), s.ref.v)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("width", [None, 128])
def test_keys_and_values_in_layouts_of_their_own(dtype, width):
    s = Setup([300, 41], [5, 30], h_kv=3, g=2, dtype=dtype, page=16, seed=48, width=width)
    # keys token by token with a gap behind each, values head by head with gaps between the pages
    k = torch.full((s.ref.k.shape[0], 16, 3, 128 + 8), math.nan, dtype=dtype, device=DEV)[..., :128].transpose(1, 2)
    v = torch.full((s.ref.k.shape[0], 4, 16, 128), math.nan, dtype=dtype, device=DEV)[:, :3]
    k.copy_(s.ref.k)
    v.copy_(s.ref.v)
    s.gpu.k, s.gpu.v = k, v
    s.check_attend()
    check_weigh(s)
    new = torch.randn((2, s.rows, 3, 128)).to(dtype)
    B.dash_paged_append(s.params(), s.gpu, new[0].to(DEV), new[1].to(DEV), s.start_gpu)
    R.append(s.ref, new[0], new[1], s.row_start)
    gen = torch.Generator().manual_seed(49)
    pos, seen = positions(s, gen)
    s.g = 1
    evict_both(s, 100, 2, 10, torch.rand(s.ref.k.shape[:3], generator=gen), pos, seen)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h_kv,lens,news", [(600, [70, 200], [1, 1]), (1030, [40], [33]), (300, [150, 20], [60, 3])])
def test_more_heads_than_the_chip_has_places(dtype, h_kv, lens, news):
    s = Setup(lens, news, h_kv=h_kv, g=1, d=64, dtype=dtype, page=16, seed=55)
    s.check_attend()
    check_weigh(s)
    gen = torch.Generator().manual_seed(56)
    pos, seen = positions(s, gen)
    evict_both(s, 32, 2, 10, torch.rand(s.ref.k.shape[:3], generator=gen), pos, seen)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_thousands_of_sequences(dtype):
    lens = [(29 * i) % 50 for i in range(3000)]
    s = Setup(lens, [i % 3 if i % 11 else 0 for i in range(3000)], h_kv=1, g=2, d=64, dtype=dtype, page=16, seed=57)
    s.check_attend()
    check_weigh(s)
    new = torch.randn((2, s.rows, 1, 64)).to(dtype)
    B.dash_paged_append(s.params(), s.gpu, new[0].to(DEV), new[1].to(DEV), s.start_gpu)
    R.append(s.ref, new[0], new[1], s.row_start)
    gen = torch.Generator().manual_seed(58)
    pos, seen = positions(s, gen)
    s.g = 1
    evict_both(s, 20, 2, 5, torch.rand(s.ref.k.shape[:3], generator=gen), pos, seen)


def test_a_given_scale():
    s = Setup([200], [4], seed=10)
    s.check_attend(scale=0.3)


def test_pages_past_four_gigabytes():
    d, page, h_kv = 128, 64, 8
    n_pages = 40000                                             # 5.2 GB each
    k = torch.zeros((n_pages, h_kv, page, d), dtype=BF, device=DEV)
    v = torch.zeros_like(k)
    small = Setup([130, 60], [2, 1], h_kv=h_kv, g=1, page=page, seed=11)
    far = n_pages - small.ref.k.shape[0]
    k[far:], v[far:] = small.gpu.k, small.gpu.v
    o, lse = small.attend()
    small.gpu = B.PagedCache(k, v, torch.where(small.gpu.table >= 0, small.gpu.table + far, small.gpu.table), small.gpu.lens)
    o2, lse2 = small.attend()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_bad_page_spoils_its_own_sequence_only(dtype):
    for m, width in ((2, None), (40, 128)):
        s = Setup([100, 90], [m, m], dtype=dtype, seed=12, width=width)
        good, _ = s.attend()
        for bad in (1 << 30, -5, s.gpu.k.shape[0]):
            s.gpu.table[0, 2] = bad
            o, _ = s.attend()
            assert torch.equal(o[m:2 * m], good[m:2 * m])


def test_lengths_and_row_starts_out_of_range_are_clamped():
    s = Setup([100, 90], [2, 2], seed=13)
    good, _ = s.attend()
    cap = s.gpu.table.shape[1] * 16
    s.gpu.lens[0] = 1 << 30
    o, _ = s.attend()
    s.gpu.lens[0] = cap                                         # the same as the whole table
    o2, _ = s.attend()
    assert torch.equal(o[2:4], good[2:4]) and torch.equal(o[:2].isnan(), o2[:2].isnan())
    s.gpu.lens[0] = -7
    o, lse = s.attend()
    assert (o[:2] == 0).all() and torch.isneginf(lse[:2]).all() and torch.equal(o[2:4], good[2:4])
    s.gpu.lens[0] = 100
    s.start_gpu = torch.tensor([-3, 2, 1 << 30], dtype=torch.int32, device=DEV)
    o, _ = s.attend()
    assert torch.equal(o, good)


def test_fp32_values_that_are_not_finite_reach_only_the_rows_that_see_them():
    s = Setup([60], [20], dtype=F32, seed=14)
    page, off = s.ref.where(0, 60)
    s.gpu.v[int(page[50]), 0, int(off[50])] = math.nan          # token 10 of the new ones, kv-head 0
    s.gpu.k[int(page[45]), 1, int(off[45])] = math.inf          # token 5, kv-head 1
    good = R.attend(s.ref, s.q, s.row_start, 2)
    o, _ = s.attend()
    clean = lambda x, w, t: ((x.double() - w).abs() <= t).all()  # noqa: E731
    assert clean(o[:10, :4], good[0][:10, :4], good[2][:10, :4]) and clean(o[:5, 4:], good[0][:5, 4:], good[2][:5, 4:])
    assert o[10:, :4].isnan().all()


# ---- weights ---------------------------------------------------------------------------------------------------------
def check_weigh(s, causal=True, last=0, seed=0, lse=None):
    gen = torch.Generator().manual_seed(seed)
    if lse is None:
        lse = R.attend(s.ref, s.q, s.row_start, s.h_kv, causal)[1].float()
    lse = torch.where(torch.isnan(lse), torch.zeros(()), lse)
    w0 = torch.rand(s.ref.k.shape[:3], generator=gen) * 0.01
    s.ref.weights = w0
    s.gpu.weights = w0.to(DEV)
    p = s.params(causal)
    ws = B.alloc_paged_workspace(p, DEV)
    ws.fill_(255)
    B.dash_paged_weigh(p, s.gpu, s.q.to(DEV), s.start_gpu, lse.to(DEV), ws, last=last)
    got = s.gpu.weights.cpu()
    want, tol = R.weigh(s.ref, s.q, s.row_start, lse, s.h_kv, causal, last=last)
    free = tol == 0
    assert torch.equal(got[free], w0[free])                     # nothing else is touched
    assert ((got.double() - want).abs() <= tol).all(), float(((got.double() - want).abs() / tol.clamp(min=1e-30)).max())
    return got


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
def test_weights_of_single_tokens(dtype, d, page):
    check_weigh(Setup(EDGE, [1] * len(EDGE), d=d, page=page, dtype=dtype, behind=math.nan, seed=20))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("last", [0, 1, 16, 1000])
def test_weights_of_chunks(dtype, causal, last):
    s = Setup([500, 20, 700, 1, 131, 0], [7, 0, 600, 1, 131, 2], h_kv=2, g=4, dtype=dtype, page=16, spare=2, behind=math.inf, seed=21)
    check_weigh(s, causal, last)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h_kv,g", [(1, 1), (3, 2), (1, 16), (8, 1)])
def test_weights_of_head_layouts(dtype, h_kv, g):
    check_weigh(Setup([300, 41, 1000], [1, 3, 90], h_kv=h_kv, g=g, d=64, dtype=dtype, page=32, layout="token", seed=22))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [1, 100])
def test_weights_of_strided_queries(dtype, new):
    s = Setup([300, 41], [new, min(new, 20)], dtype=dtype, page=32, layout="token", seed=33)
    lse = R.attend(s.ref, s.q, s.row_start, 2)[1].float()
    want = check_weigh(s, lse=lse)
    p = s.params()
    fused = torch.full((s.rows, 12, 128 + 8), math.nan, dtype=dtype, device=DEV)
    by_head = torch.full((8, s.rows, 128), math.nan, dtype=dtype, device=DEV)
    for q in (fused[:, 4:, 8:], by_head.transpose(0, 1)):
        q.copy_(s.q)
        s.gpu.weights = s.ref.weights.to(DEV)
        B.dash_paged_weigh(p, s.gpu, q, s.start_gpu, lse.to(DEV), B.alloc_paged_workspace(p, DEV))
        assert torch.equal(s.gpu.weights.cpu(), want)


def test_weights_of_a_long_cache_and_a_large_batch():
    check_weigh(Setup([30000], [40], h_kv=1, g=4, page=64, seed=23))
    lens = [(37 * i) % 400 for i in range(150)]
    check_weigh(Setup(lens, [i % 3 for i in range(150)], h_kv=1, g=2, d=64, page=16, seed=24))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_weights_of_rows_that_see_nothing(dtype):
    check_weigh(Setup([5, 0, 20], [9, 4, 30], dtype=dtype, seed=25))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_rows_outside_the_window_weigh_nothing_whatever_they_hold(dtype):
    s = Setup([200], [30], dtype=dtype, seed=26)
    lse = R.attend(s.ref, s.q, s.row_start, 2)[1].float()
    want = check_weigh(s, last=8, lse=lse)
    s.q[:22] = math.nan
    lse[:22] = math.nan
    w0 = s.ref.weights
    s.gpu.weights = w0.to(DEV)
    p = s.params()
    B.dash_paged_weigh(p, s.gpu, s.q.to(DEV), s.start_gpu, lse.to(DEV), B.alloc_paged_workspace(p, DEV), last=8)
    assert torch.equal(s.gpu.weights.cpu(), want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("m,bad", [(2, 0), (30, 5), (130, 77)])
def test_weights_a_row_that_is_nan_reaches_only_the_tokens_it_sees(dtype, m, bad):
    s = Setup([200], [m], dtype=dtype, seed=31)
    lse = R.attend(s.ref, s.q, s.row_start, 2)[1].float()
    s.ref.weights = torch.zeros(s.ref.k.shape[:3])
    q, l = s.q.clone(), lse.clone()
    q[bad], l[bad] = 0.0, math.inf                              # the row left out
    want, tol = R.weigh(s.ref, q, s.row_start, l, 2)
    s.q[bad], lse[bad] = math.nan, math.nan
    s.gpu.weights = s.ref.weights.to(DEV)
    p = s.params()
    B.dash_paged_weigh(p, s.gpu, s.q.to(DEV), s.start_gpu, lse.to(DEV), B.alloc_paged_workspace(p, DEV))
    page, off = s.ref.where(0, 200)
    got, want, tol = (x[page, :, off] for x in (s.gpu.weights.cpu(), want, tol))
    seen = 200 - m + bad + 1
    assert got[:seen].isnan().all()
    assert ((got[seen:].double() - want[seen:]).abs() <= tol[seen:]).all()


@pytest.mark.parametrize("last", [0, 2])
@pytest.mark.parametrize("d,g", [(128, 4), (64, 8), (128, 1)])
@pytest.mark.parametrize("news", [[70] + [1] * 30, [1, 2, 0, 33] + [3] * 36, [0] * 20 + [25] + [0] * 9, [5] * 12])
def test_weights_of_long_and_short_pieces_in_one_call(last, d, g, news):
    check_weigh(Setup([(83 * i) % 500 + news[i] for i in range(len(news))], news, h_kv=2, g=g, d=d, page=16, behind=math.nan, seed=42), last=last)


def test_weights_of_pages_that_sequences_share():
    s = Setup([300, 280], [1, 2], page=16, seed=28)
    s.ref.table[1, :17] = s.ref.table[0, :17]                   # 272 tokens in common
    s.gpu.table.copy_(s.ref.table)
    check_weigh(s)


def test_a_bad_page_gets_no_weights():
    s = Setup([100, 90], [2, 2], seed=27)
    lse = R.attend(s.ref, s.q, s.row_start, 2)[1].float()
    s.gpu.weights = torch.zeros(s.ref.k.shape[:3], device=DEV)
    s.gpu.table[0, 2] = -1
    unused = sorted(set(range(s.ref.k.shape[0])) - set(s.gpu.table[s.gpu.table >= 0].tolist()))
    p = s.params()
    B.dash_paged_weigh(p, s.gpu, s.q.to(DEV), s.start_gpu, lse.to(DEV), B.alloc_paged_workspace(p, DEV))
    assert (s.gpu.weights[unused] == 0).all() and (s.gpu.weights > 0).any()


# ---- append ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,page,layout,h_kv", [(64, 16, "head", 3), (128, 64, "token", 2), (128, 16, "token", 9)])
@pytest.mark.parametrize("evicting", [True, False])
def test_append(dtype, d, page, layout, h_kv, evicting):
    s = Setup([40, 0, 5, 100, 17, 64], [1, 0, 9, 100, 17, 1], h_kv=h_kv, g=1, d=d, page=page, dtype=dtype, spare=2, layout=layout, seed=30)
    gen = torch.Generator().manual_seed(31)
    new = torch.randn((2, s.rows, h_kv, d), generator=gen).to(dtype)
    if evicting:
        s.ref.weights, s.ref.pos = torch.rand(s.ref.k.shape[:3], generator=gen), torch.full(s.ref.k.shape[:3], -9, dtype=torch.int32)
        s.ref.seen = s.ref.lens + 1000
        s.gpu.weights, s.gpu.pos, s.gpu.seen = s.ref.weights.to(DEV), s.ref.pos.to(DEV), s.ref.seen.to(DEV)
    s.ref.table[3, 3 if page == 16 else 0] = s.gpu.table[3, 3 if page == 16 else 0] = s.ref.k.shape[0]     # no page
    big = torch.zeros((s.rows, h_kv, 2, d), dtype=dtype, device=DEV)
    big[:, :, 0], big[:, :, 1] = new[0].to(DEV), new[1].to(DEV)
    B.dash_paged_append(s.params(), s.gpu, big[:, :, 0], big[:, :, 1], s.start_gpu)
    R.append(s.ref, new[0], new[1], s.row_start)
    assert torch.equal(s.gpu.k.cpu(), s.ref.k) and torch.equal(s.gpu.v.cpu(), s.ref.v)
    if evicting:
        assert torch.equal(s.gpu.weights.cpu(), s.ref.weights) and torch.equal(s.gpu.pos.cpu(), s.ref.pos)


def test_append_of_more_rows_than_a_launch_has_threads_for():
    # a wave a row: 64 (2^26 + 5) threads.  The rows share one row of memory; the second sequence is shorter than its rows, so its last three are written.
    n, c = (1 << 26) + 5, B.PagedCache.allocate(2, 1, 2, 16, 64, 1, DEV)
    c.table.copy_(torch.tensor([[1], [0]]))
    c.lens.copy_(torch.tensor([5, 3]))
    row = torch.randn((2, 1, 1, 64), dtype=BF, device=DEV)
    start = torch.tensor([0, 5, n], dtype=torch.int32, device=DEV)
    B.dash_paged_append(B.make_paged_params(c, n, 1), c, row[0].expand(n, 1, 64), row[1].expand(n, 1, 64), start)
    for x, y in ((c.k, row[0]), (c.v, row[1])):
        want = torch.zeros_like(x)
        want[1, 0, :5] = want[0, 0, :3] = y[0, 0]
        assert torch.equal(x, want)


def test_append_positions_without_seen_and_a_large_batch():
    lens = [1 + (37 * i) % 90 for i in range(150)]
    s = Setup(lens, [min(n, i % 4) for i, n in enumerate(lens)], h_kv=1, g=1, d=64, page=16, seed=32)
    s.ref.pos = torch.full(s.ref.k.shape[:3], -9, dtype=torch.int32)
    s.gpu.pos = s.ref.pos.to(DEV)
    new = torch.randn((2, s.rows, 1, 64)).to(BF)
    B.dash_paged_append(s.params(), s.gpu, new[0].to(DEV), new[1].to(DEV), s.start_gpu)
    R.append(s.ref, new[0], new[1], s.row_start)
    assert torch.equal(s.gpu.k.cpu(), s.ref.k) and torch.equal(s.gpu.v.cpu(), s.ref.v) and torch.equal(s.gpu.pos.cpu(), s.ref.pos)


# ---- eviction --------------------------------------------------------------------------------------------------------
def evict_both(s, budget, sinks, recent, weights, pos, seen, with_src=True):
    s.ref.weights, s.ref.pos, s.ref.seen = weights, pos, seen
    s.gpu.weights, s.gpu.pos, s.gpu.seen = weights.to(DEV), pos.to(DEV), seen.to(DEV)
    p = s.params()
    ws = B.alloc_paged_workspace(p, DEV, evict=True)
    ws.fill_(255)
    src = torch.full((len(s.ref.lens), s.h_kv, budget), 5, dtype=torch.int32, device=DEV) if with_src else None
    B.dash_paged_evict(p, s.gpu, budget, ws, sinks=sinks, recent=recent, src=src)
    want = R.evict(s.ref, budget, sinks, recent)
    if with_src:
        assert torch.equal(src.cpu(), want)
    assert torch.equal(s.gpu.lens.cpu(), s.ref.lens)
    for x, y in ((s.gpu.k, s.ref.k), (s.gpu.v, s.ref.v), (s.gpu.pos, s.ref.pos)):
        assert torch.equal(x.cpu(), y)
    assert torch.equal(s.gpu.weights.cpu().view(torch.int32), s.ref.weights.view(torch.int32))


def positions(s, gen, extra=50):
    pos = torch.zeros(s.ref.k.shape[:3], dtype=torch.int32)
    for b, n in enumerate(s.ref.lens.tolist()):
        page, off = s.ref.where(b, n)
        for h in range(s.h_kv):
            pos[page, h, off] = torch.randperm(n + extra, generator=gen)[:n].to(torch.int32)
    return pos, s.ref.lens + extra


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,page,layout", [(64, 16, "head"), (128, 64, "token"), (128, 128, "head")])
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (100, 4, 20), (64, 32, 32), (255, 0, 255), (300, 0, 10), (2500, 5, 700)])
def test_evict(dtype, d, page, layout, budget, sinks, recent):
    s = Setup([0, 1, 100, 101, 257, 2300, 300, 4097], [1] * 8, h_kv=3, g=1, d=d, page=page, dtype=dtype, layout=layout, seed=40)
    gen = torch.Generator().manual_seed(41)
    w = torch.randn(s.ref.k.shape[:3], generator=gen).exp()
    pos, seen = positions(s, gen)
    evict_both(s, budget, sinks, recent, w, pos, seen)


@pytest.mark.parametrize("kind", ["all equal", "zeros and ones", "special", "negative", "near"])
def test_evict_ties_and_special_weights(kind):
    s = Setup([1500, 1100, 700], [1] * 3, h_kv=2, g=1, d=64, page=16, seed=42)
    gen = torch.Generator().manual_seed(43)
    shape = s.ref.k.shape[:3]
    w = {"all equal": torch.ones(shape), "zeros and ones": (torch.rand(shape, generator=gen) < 0.3).float(),
         "special": torch.tensor([0.0, -0.0, math.nan, math.inf, 1e-40, 1.0, -1.0])[torch.randint(0, 7, shape, generator=gen)],
         "negative": torch.randn(shape, generator=gen),
         "near": 1.0 + torch.randint(0, 3, shape, generator=gen) * 2.0 ** -23}[kind]
    pos, seen = positions(s, gen)
    evict_both(s, 600, 3, 50, w, pos, seen)


# more than 2048 keys that share their leading bits with the one looked for, and others
@pytest.mark.parametrize("budget", [600, 3000, 4999, 8000])
@pytest.mark.parametrize("kind", ["all equal", "zeros and ones", "near", "any"])
def test_evict_ties_of_thousands(kind, budget):
    s = Setup([8192, 5000, 2100], [1] * 3, h_kv=2, g=1, d=64, page=16, seed=50)
    gen = torch.Generator().manual_seed(51)
    shape = s.ref.k.shape[:3]
    w = {"all equal": torch.full(shape, 0.25), "zeros and ones": (torch.rand(shape, generator=gen) < 0.4).float(),
         "near": 1.0 + torch.randint(0, 2048, shape, generator=gen) * 2.0 ** -23, "any": torch.randn(shape, generator=gen).exp()}[kind]
    pos, seen = positions(s, gen)
    evict_both(s, budget, 3, 50, w, pos, seen)


@pytest.mark.parametrize("longest", [700, 9000])                # both ways to select
@pytest.mark.parametrize("bad", [-1, 1 << 30, None])
def test_evict_with_a_bad_page_leaves_the_others_alone(longest, bad):
    s = Setup([600, 500, longest], [1] * 3, h_kv=2, g=1, d=64, page=16, seed=52)
    gen = torch.Generator().manual_seed(53)
    w = torch.randn(s.ref.k.shape[:3], generator=gen).exp()
    pos, seen = positions(s, gen)
    mine = s.ref.table[0][s.ref.table[0] >= 0].long()
    s.ref.weights, s.ref.pos, s.ref.seen = w, pos, seen
    s.gpu.weights, s.gpu.pos, s.gpu.seen = w.to(DEV), pos.to(DEV), seen.to(DEV)
    for i in (1, 7, 30, 37):                                    # before the budget, behind it, the last one
        s.gpu.table[0, i] = s.ref.k.shape[0] if bad is None else bad
    p = s.params()
    ws = B.alloc_paged_workspace(p, DEV, evict=True)
    ws.fill_(255)
    B.dash_paged_evict(p, s.gpu, 300, ws, sinks=2, recent=20)
    s.ref.lens[0] = 0                                           # the others by themselves
    R.evict(s.ref, 300, 2, 20)
    others = torch.ones(s.ref.k.shape[0], dtype=torch.bool)
    others[mine] = False
    assert s.gpu.lens.tolist() == [300, 300, 300]
    for x, y in ((s.gpu.k, s.ref.k), (s.gpu.v, s.ref.v), (s.gpu.pos, s.ref.pos), (s.gpu.weights, s.ref.weights)):
        assert torch.equal(x.cpu()[others], y[others])


@pytest.mark.parametrize("n", [100, 9000])                      # both ways to select
def test_evict_a_budget_near_the_largest_number(n):
    # src has a slot for every token of the budget: 2^31 - 1 of them
    s = Setup([n], [1], h_kv=1, g=1, d=64, page=16, seed=54)
    s.gpu.weights, s.gpu.pos, s.gpu.seen = (torch.zeros(s.ref.k.shape[:3], dtype=t, device=DEV) for t in (F32, torch.int32, torch.int32))
    s.gpu.seen = s.gpu.lens.clone()
    p = s.params()
    budget = (1 << 31) - 1
    src = torch.full((1, 1, budget), 5, dtype=torch.int32, device=DEV)
    B.dash_paged_evict(p, s.gpu, budget, B.alloc_paged_workspace(p, DEV, evict=True), src=src)
    assert s.gpu.lens.item() == n and torch.equal(src[0, 0, :n].cpu(), torch.arange(n, dtype=torch.int32))
    assert all(bool((x == -1).all()) for x in src[0, 0, n:].split(1 << 28))
    assert torch.equal(s.gpu.k.cpu(), s.ref.k) and torch.equal(s.gpu.v.cpu(), s.ref.v)


def test_evict_without_src_and_with_everything_protected():
    s = Setup([500], [1], h_kv=2, g=1, d=64, page=16, seed=44)
    gen = torch.Generator().manual_seed(45)
    w = torch.rand(s.ref.k.shape[:3], generator=gen)
    pos = torch.zeros(s.ref.k.shape[:3], dtype=torch.int32)     # every token has position 0: more are protected than stay
    evict_both(s, 200, 1, 0, w, pos, s.ref.lens.clone(), with_src=False)


@pytest.mark.parametrize("budget", [32768, 500, 69000, 4111, 4096, 1])
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("page", [16, 64])
def test_evict_long_sequences(budget, ties, page):
    s = Setup([70000, 33000, 32768, 0, 4112], [1, 1, 1, 1, 1], h_kv=1, g=1, d=64, page=page, seed=46)
    gen = torch.Generator().manual_seed(47)
    w = torch.randn(s.ref.k.shape[:3], generator=gen).exp()
    if ties:
        w = (w > 1.5).float()
    pos, seen = positions(s, gen)
    evict_both(s, budget, min(4, budget), min(100, budget - min(4, budget)), w, pos, seen)


def test_evict_more_caches_than_workgroups_fit():
    s = Setup([(11 * i) % 60 for i in range(300)], [1] * 300, h_kv=8, g=1, d=64, page=16, seed=48)
    gen = torch.Generator().manual_seed(49)
    pos, seen = positions(s, gen)
    evict_both(s, 32, 2, 8, torch.rand(s.ref.k.shape[:3], generator=gen), pos, seen)


# ---- together --------------------------------------------------------------------------------------------------------
class Server:
    """Prompts in chunks beside decoding sequences on caches held to a budget: every call of a step on the GPU, the same steps
    plainly on the CPU."""

    def __init__(self, dtype, seed, batch=3, h_kv=2, g=2, d=64, page=16, budget=96, slots=160):
        self.dtype, self.h_kv, self.g, self.d, self.budget = dtype, h_kv, g, d, budget
        self.gen = torch.Generator().manual_seed(seed)
        per = slots // page
        self.c = B.PagedCache.allocate(batch, h_kv, batch * per, page, d, per, DEV, dtype, evicting=True)
        self.c.table.copy_(torch.randperm(batch * per, generator=self.gen).view(batch, per))
        self.ref = R.Cache(*(x.cpu().clone() for x in (self.c.k, self.c.v, self.c.table, self.c.lens, self.c.weights, self.c.pos, self.c.seen)))
        self.ws = self.ws_e = None
        self.mid = torch.zeros_like(self.c.weights)

    def new_rows(self, news):
        rand = lambda h: torch.randn((sum(news), h, self.d), generator=self.gen).to(self.dtype)  # noqa: E731
        start = [0]
        for m in news:
            start.append(start[-1] + m)
        return rand(self.h_kv * self.g) * 2, rand(self.h_kv), rand(self.h_kv), torch.tensor(start, dtype=torch.int32)

    def grow(self, start):
        m = start[1:] - start[:-1]
        self.ref.lens += m
        self.ref.seen += m

    def calls(self, p, q, k, v, start, o, lse):
        B.dash_paged_append(p, self.c, k, v, start)
        B.dash_paged_attend(p, self.c, q, start, o, self.ws, lse=lse)
        B.dash_paged_weigh(p, self.c, q, start, lse, self.ws)
        self.mid.copy_(self.c.weights)
        B.dash_paged_evict(p, self.c, self.budget, self.ws_e, sinks=2, recent=16)

    def step(self, news):
        q, k, v, start = self.new_rows(news)
        self.grow(start)
        self.c.lens.copy_(self.ref.lens)
        self.c.seen.copy_(self.ref.seen)
        p = B.make_paged_params(self.c, q.shape[0], self.h_kv * self.g)
        if self.ws is None:
            self.ws, self.ws_e = B.alloc_paged_workspace(p, DEV), B.alloc_paged_workspace(p, DEV, evict=True)
        o, lse = torch.empty_like(q, device=DEV), torch.empty(q.shape[:2], device=DEV)
        self.calls(p, q.to(DEV), k.to(DEV), v.to(DEV), start.to(DEV), o, lse)
        self.compare(q, k, v, start, o, lse)

    def compare(self, q, k, v, start, o, lse):
        R.append(self.ref, k, v, start)
        want, wl, tol, ltol = R.attend(self.ref, q, start, self.h_kv)
        assert ((o.cpu().double() - want).abs() <= tol).all() and ((lse.cpu().double() - wl).abs() <= ltol).all()
        w, tol = R.weigh(self.ref, q, start, lse.cpu(), self.h_kv)
        assert ((self.mid.cpu().double() - w).abs() <= tol).all()
        self.ref.weights = self.mid.cpu().clone()               # which tokens stay goes by the weights as they were added up
        R.evict(self.ref, self.budget, 2, 16)
        for x, y in ((self.c.k, self.ref.k), (self.c.v, self.ref.v), (self.c.pos, self.ref.pos), (self.c.weights, self.ref.weights),
                     (self.c.lens, self.ref.lens)):
            assert torch.equal(x.cpu(), y)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_serving_loop(dtype):
    s = Server(dtype, 50)
    for news in ([60, 0, 1], [60, 33, 1], [40, 50, 1], [1, 60, 1], [1, 1, 30], [1, 1, 1], [1, 1, 1], [5, 0, 64], [1, 1, 1], [64, 64, 64]):
        s.step(news)
    assert (s.c.lens == s.budget).all()


def test_a_step_in_a_captured_graph():
    s = Server(BF, 51)
    for news in ([60, 70, 80], [50, 40, 1]):
        s.step(news)
    q, k, v, start = s.new_rows([1, 1, 1])
    p = B.make_paged_params(s.c, 3, s.h_kv * s.g)
    buf = [x.to(DEV) for x in (q, k, v, start)]
    o, lse = torch.empty_like(buf[0]), torch.empty(q.shape[:2], device=DEV)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        s.calls(p, *buf, o, lse)
    torch.cuda.synchronize()
    for i in range(4):
        if i == 2:
            s.step([30, 1, 64])                                 # the program's own eager work between the replays
        q, k, v, start = s.new_rows([1, 1, 1])
        s.grow(start)
        s.c.lens.copy_(s.ref.lens)
        s.c.seen.copy_(s.ref.seen)
        for x, y in zip(buf, (q, k, v, start)):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        s.compare(q, k, v, start, o, lse)


def test_calls_on_two_streams_with_a_workspace_each():
    a, b = (Setup([4000, 900], [2, 50], h_kv=2, g=4, page=64, seed=60 + i) for i in range(2))
    want = [x.attend() for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ins = [(x.params(), x.q.to(DEV)) for x in (a, b)]
    outs = [torch.empty_like(q) for _, q in ins]
    wss = [B.alloc_paged_workspace(p, DEV) for p, _ in ins]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, st, (p, q), o, ws in zip((a, b), streams, ins, outs, wss):
            with torch.cuda.stream(st):
                B.dash_paged_attend(p, x.gpu, q, x.start_gpu, o, ws)
    torch.cuda.synchronize()
    for o, (w, _) in zip(outs, want):
        assert torch.equal(o.cpu(), w)


def test_the_same_call_gives_the_same_bits():
    s = Setup([9000, 100, 3000], [1, 60, 300], h_kv=2, g=4, page=32, seed=70)
    a, b = s.attend(), s.attend()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    lse = a[1]
    x, y = (check_weigh(s, lse=lse) for _ in range(2))
    assert torch.equal(x, y)
