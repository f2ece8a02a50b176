"""The paged cache in 4 bits against its definition in 64 bits (tests/paged4_ref.py and tests/paged_ref.py, which derive the bounds)."""
import math

import pytest
import torch

import paged4_ref as R
import paged_ref as P
from paper_2605_18753_amd import binding as B
from test_gpu_rotary import Fresh, check, draws

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def held(x):
    return R.values(*R.quantise(x))


# ---- append and unpack -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", [None, "halves", "adjacent"])
@pytest.mark.parametrize("d,rot,h_q,h_kv,page", [(64, 64, 4, 2, 16), (128, 128, 32, 8, 64), (128, 48, 3, 3, 32), (64, 16, 16, 1, 16), (128, 80, 5, 5, 16)])
def test_append(dtype, layout, d, rot, h_q, h_kv, page):
    s = Fresh([40, 5, 1, 33, 0, 2], [9, 5, 1, 33, 0, 6], h_q, h_kv, d, page, dtype, spare=2, seed=21, missing=((3, 0, 999), (0, 1 if page < 40 else 0, -1)),
              seen=[1000, 7, 70001, 2 ** 30, 5, 9])
    c = B.PagedCache4.allocate(6, h_kv, s.n_pages, page, d, s.table.shape[1], DEV)
    gen = torch.Generator().manual_seed(3)
    for x in (c.k_codes, c.v_codes, c.k_scales, c.v_scales):
        x.copy_(torch.randint(7, 250, x.shape, generator=gen, dtype=torch.uint8))
    before = [x.cpu() for x in (c.k_codes, c.k_scales, c.v_codes, c.v_scales)]
    c.table.copy_(s.table)
    c.lens.copy_(torch.tensor(s.lens))
    c.seen = s.seen.to(DEV)
    p = B.make_paged4_params(c, s.rows, h_q, dtype=dtype)
    kw, q_out = {}, torch.full_like(s.q, 77.0, device=DEV)
    if layout:
        kw = dict(rotary=B.make_rotary(rot, DEV, layout=layout, mscale=0.75), q=s.q.to(DEV), q_out=q_out)
    B.dash_paged4_append(p, c, s.k_new.to(DEV), s.v_new.to(DEV), s.row_start.to(DEV), **kw)
    theta = R.thetas(rot)
    rows = [x[0] for x in s.places]
    if layout:
        at = torch.tensor([x[3] for x in s.places])
        check(q_out.cpu()[rows], s.q[rows], at[:, None], theta, layout, 0.75)
        assert (q_out[[i for i in range(s.rows) if i not in set(rows)]] == 77).all()
    after = [x.cpu() for x in (c.k_codes, c.k_scales, c.v_codes, c.v_scales)]
    done = list(s.written())
    assert 0 < len(done) < len(rows) < s.rows
    for row, b, slot, position, pg, off in done:
        k = R.turn(s.k_new[row], torch.tensor(position), theta, layout, 0.75)[0] if layout else s.k_new[row]
        for x, i in ((k, 0), (s.v_new[row], 2)):
            assert torch.equal(R.values(after[i][pg, :, off], after[i + 1][pg, :, off]), held(x))
        for x, y in zip(after, before):
            x[pg, :, off] = y[pg, :, off]
    assert all(torch.equal(x, y) for x, y in zip(after, before))  # nothing else is touched


@pytest.mark.parametrize("dtype", [BF, F32])
def test_every_kind_of_number(dtype):
    """Ties, the border of the scale, zeros, numbers that are not finite, the largest and smallest, and every bf16 beside a largest of its size."""
    d, rows = 64, []
    tie = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    for top in (4.0, 6.0, 7.25, 7.28125, 7.96875, 8.0, 4.03125):
        for scale in (1.0, 2.0 ** -20, 2.0 ** 100, 2.0 ** -119):
            rows.append([top * scale] + [x * scale for t in tie for x in (t, -t, t * (1 + 2 ** -7), t * (1 - 2 ** -8))] + [0.0, -0.0, top * scale / 2])
    rows += [[0.0] * 32, [-0.0] * 32, [2.0 ** -130] * 32, [3.0e38] * 32, [-3.3895e38] + [1.7e38] * 31, [2.0 ** -126] * 16 + [2.0 ** -121] * 16]
    rows += [[1.0] * 31 + [math.nan], [math.inf] + [1.0] * 31, [1.0] * 15 + [-math.inf] + [2.0] * 16]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype)
    bits = torch.arange(0, 1 << 15, dtype=torch.int32).to(torch.int16).view(BF)        # all that are not negative
    every = bits.view(-1, 32)[torch.isfinite(bits.view(-1, 32)).all(-1)].to(dtype)
    lead = torch.cat((every[:, 31:] * 3, every[:, 1:]), 1)
    x = torch.cat((x, every, -every, torch.where(torch.isfinite(lead), lead, torch.zeros((), dtype=dtype))))
    x = torch.cat((x, x.flip(0)), 1)[:, None]                    # [rows, 1, 64]
    n = x.shape[0]
    c = B.PagedCache4.allocate(1, 1, -(-n // 64), 64, d, -(-n // 64), DEV)
    c.table.copy_(torch.arange(c.table.shape[1])[None])
    c.lens.fill_(n)
    p = B.make_paged4_params(c, n, 1, dtype=dtype)
    B.dash_paged4_append(p, c, x.to(DEV), x.flip(0).contiguous().to(DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV))
    for codes, scales, want in ((c.k_codes, c.k_scales, held(x)), (c.v_codes, c.v_scales, held(x.flip(0)))):
        got = R.values(codes.cpu(), scales.cpu()).reshape(-1, 1, d)[:n]
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        bad = ~((got == want) | torch.isnan(want))
        assert not bad.any(), (x[bad.any(-1).any(-1)][:3], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_unpack_every_code_and_scale(dtype, d):
    gen = torch.Generator().manual_seed(4)
    c = B.PagedCache4.allocate(1, 3, 9, 16, d, 9, DEV)
    codes = torch.randint(0, 256, c.k_codes.shape, generator=gen, dtype=torch.uint8)
    scales = torch.randint(7, 253, c.k_scales.shape, generator=gen, dtype=torch.uint8)
    codes.view(-1)[:256] = torch.arange(256, dtype=torch.uint8)
    scales.view(-1)[:246], scales.view(-1)[246:250] = torch.arange(7, 253, dtype=torch.uint8), 255
    c.k_codes.copy_(codes), c.k_scales.copy_(scales), c.v_codes.copy_(codes.flip(0)), c.v_scales.copy_(scales.flip(0))
    p = B.make_paged4_params(c, 1, 3, dtype=dtype)
    k, v = (torch.full((9, 3, 16, d), 77.0, dtype=dtype, device=DEV) for _ in range(2))
    B.dash_paged4_unpack(p, c, k, v)
    for got, want in ((k, R.values(codes, scales)), (v, R.values(codes.flip(0), scales.flip(0)))):
        got = got.cpu().double()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_append_and_unpack_of_codes_in_another_layout(dtype, d):
    """Heads inside of tokens, with room behind each row of codes; K and V in layouts of their own; packed rows that are slices of one tensor.  Rows of several
    workgroups lie side by side: every byte is its own row's."""
    h_kv, page, n = 3, 32, 700
    n_pages = -(-n // page) + 1
    wide = torch.full((n_pages, page, h_kv, d // 2 + 16), 171, dtype=torch.uint8, device=DEV)
    c = B.PagedCache4.allocate(1, h_kv, n_pages, page, d, n_pages, DEV)
    c.k_codes = wide[..., :d // 2].transpose(1, 2)
    c.table.copy_(torch.randperm(n_pages, generator=torch.Generator().manual_seed(1))[None])
    c.lens.fill_(n)
    fused = draws(30)(n, 4 * h_kv, d).to(dtype).to(DEV)
    q, k, v = fused[:, :2 * h_kv], fused[:, 2 * h_kv:3 * h_kv], fused[:, 3 * h_kv:]
    before = fused.cpu().clone()
    p = B.make_paged4_params(c, n, 2 * h_kv, dtype=dtype)
    r = B.make_rotary(d, DEV)
    B.dash_paged4_append(p, c, k, v, torch.tensor([0, n], dtype=torch.int32, device=DEV), rotary=r, q=q, q_out=q)
    kp, vp = (torch.full((n_pages, h_kv, page, d), 77.0, dtype=dtype, device=DEV) for _ in range(2))
    B.dash_paged4_unpack(p, c, kp, vp)
    assert (wide[..., d // 2:] == 171).all()
    at = torch.arange(n)
    where = c.table[0].cpu().long()[at // page], at % page
    turned = R.turn(before[:, 2 * h_kv:3 * h_kv], at[:, None], R.thetas(d), "halves")[0]
    assert torch.equal(kp.cpu().double()[where[0], :, where[1]], held(turned))
    assert torch.equal(vp.cpu().double()[where[0], :, where[1]], held(before[:, 3 * h_kv:]))
    check(q.cpu(), before[:, :2 * h_kv], at[:, None], R.thetas(d), "halves")
    assert torch.equal(fused.cpu()[:, 2 * h_kv:], before[:, 2 * h_kv:])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_queries_keys_and_values_of_each_head_side_by_side(dtype):
    """Slices [n, h, (q, k, v), d] of one projection, q turned in place, by an append into pages of either kind and by the call that turns alone."""
    h, d, n, page = 4, 128, 150, 16
    each = draws(34)(n, h, 3, d).to(dtype)
    at, theta = torch.arange(n)[:, None], R.thetas(d)
    turned = R.turn(each[:, :, 1], at, theta, "halves")[0]
    r = B.make_rotary(d, DEV)
    start = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    for four in (True, False):
        g = each.to(DEV)
        q, k, v = g.unbind(2)
        c = B.PagedCache4.allocate(1, h, 10, page, d, 10, DEV) if four else B.PagedCache.allocate(1, h, 10, page, d, 10, DEV, dtype=dtype)
        c.table.copy_(torch.arange(10)[None])
        c.lens.fill_(n)
        if four:
            p = B.make_paged4_params(c, n, h, dtype=dtype)
            B.dash_paged4_append(p, c, k, v, start, rotary=r, q=q, q_out=q)
            kp, vp = (torch.zeros((10, h, page, d), dtype=dtype, device=DEV) for _ in range(2))
            B.dash_paged4_unpack(p, c, kp, vp)
            got = kp.cpu().double().transpose(0, 1).reshape(h, -1, d)[:, :n].transpose(0, 1)
            assert torch.equal(got, held(turned))
        else:
            p = B.make_paged_params(c, n, h)
            B.dash_paged_append_rotary(p, c, r, k, v, start, q=q, q_out=q)
            check(c.k.cpu().transpose(0, 1).reshape(h, -1, d)[:, :n].transpose(0, 1), each[:, :, 1], at, theta, "halves")
        check(q.cpu(), each[:, :, 0], at, theta, "halves")
        assert torch.equal(g.cpu()[:, :, 1:], each[:, :, 1:])
    g = each.to(DEV)[None]
    q, k, _ = (x.transpose(1, 2) for x in g.unbind(3))
    B.dash_rotary(r, q, q, k, k)
    for i in (0, 1):
        check(g[0, :, :, i].cpu(), each[:, :, i], at, theta, "halves")
    assert torch.equal(g.cpu()[0, :, :, 2], each[:, :, 2])


# ---- attention -------------------------------------------------------------------------------------------------------
class Setup4:
    """A cache in 4 bits on the GPU and its values on the CPU.  behind: what the pages hold behind the sequences' ends (NaN: blocks that are NaN)."""

    def __init__(self, lens, news, h_kv=2, g=4, d=128, page=16, dtype=BF, seed=0, spare=0, behind=None, layout="head", qscale=1.0, width=None):
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
        per = [-(-n // page) for n in lens]
        n_pages = sum(per) + 2
        ids = torch.randperm(n_pages, generator=gen)[:sum(per)].tolist()
        width = width or max(max(per), 1)
        table = torch.full((len(lens), width), -1, dtype=torch.int32)
        at = 0
        for b, k in enumerate(per):
            table[b, :k] = torch.tensor(ids[at:at + k], dtype=torch.int32)
            at += k
        used = torch.zeros((n_pages, page), dtype=torch.bool)
        for b, n in enumerate(lens):
            i = torch.arange(n)
            used[table[b].long()[i // page], i % page] = True
        self.codes = []
        for _ in range(2):
            codes, scales = R.quantise(rand(n_pages, h_kv, page, d)) if n_pages * h_kv * page * d < 1 << 23 else self.cheap(gen, (n_pages, h_kv, page, d))
            if behind is not None:
                codes = torch.where(used[:, None, :, None], codes, torch.full((), 0x77, dtype=torch.uint8))
                scales = torch.where(used[:, None, :, None], scales, torch.full((), 255, dtype=torch.uint8))
            self.codes += [codes, scales]
        start = [0]
        for m in news:
            start.append(start[-1] + m)
        self.row_start = torch.tensor(start, dtype=torch.int32)
        self.rows = start[-1] + spare
        self.q = (qscale * rand(max(self.rows, 1), h_kv * g, d)).to(dtype)
        self.h_kv, self.g, self.dtype, self.lens = h_kv, g, dtype, torch.tensor(lens, dtype=torch.int32)
        self.table, self.layout = table, layout
        self.start_gpu = self.row_start.to(DEV)
        self.place()

    @staticmethod
    def cheap(gen, shape):
        """Large caches: codes drawn as such."""
        return (torch.randint(0, 256, (*shape[:-1], shape[-1] // 2), generator=gen, dtype=torch.uint8),
                torch.randint(124, 127, (*shape[:-1], shape[-1] // 32), generator=gen, dtype=torch.uint8))

    def place(self):
        kc, ks, vc, vs = self.codes
        self.ref = P.Cache(R.values(kc, ks).float(), R.values(vc, vs).float(), self.table, self.lens)
        on = [x.to(DEV) for x in self.codes]
        if self.layout == "token":                               # heads inside of tokens
            on[0], on[2] = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (on[0], on[2]))
        self.gpu = B.PagedCache4(*on, self.table.to(DEV), self.lens.to(DEV))

    def params(self, causal=True, scale=0.0):
        return B.make_paged4_params(self.gpu, self.q.shape[0], self.h_kv * self.g, dtype=self.dtype, causal=causal, scale=scale)

    def attend(self, causal=True, scale=0.0, q=None):
        p = self.params(causal, scale)
        q = self.q.to(DEV) if q is None else q
        o = torch.full(q.shape, 77.0, dtype=q.dtype, device=DEV)
        lse = torch.full(q.shape[:2], 77.0, dtype=F32, device=DEV)
        ws = B.alloc_paged4_workspace(p, DEV)
        ws.fill_(255)                                            # NaN everywhere
        B.dash_paged4_attend(p, self.gpu, q, self.start_gpu, o, ws, lse=lse)
        torch.cuda.synchronize()
        return o.cpu(), lse.cpu()

    def check(self, causal=True, scale=0.0, q=None):
        o, lse = self.attend(causal, scale, q)
        want, wl, tol, ltol = P.attend(self.ref, self.q, self.row_start, self.h_kv, causal, scale or None)
        # weights below 2^-126 of a row's largest come out as 0: all that a row has where the numbers of its heaviest keys are held as 0
        tol = tol + float(self.lens.max()) * 2.0 ** -126 * float(self.ref.v[torch.isfinite(self.ref.v)].abs().max())
        own = int(self.row_start[-1])
        assert (o[own:].float() == 77).all() and (lse[own:] == 77).all()          # rows of no sequence
        o, lse, want, wl, tol, ltol = (x[:own] for x in (o, lse, want, wl, tol, ltol))
        assert torch.equal(torch.isneginf(lse), torch.isneginf(wl))
        seen = ~torch.isneginf(wl)
        assert ((lse.double() - wl).abs()[seen] <= ltol[seen]).all(), float(((lse.double() - wl).abs() / ltol)[seen].max())
        assert not torch.isnan(o).any()
        assert ((o.double() - want).abs() <= tol).all(), float(((o.double() - want).abs() / tol.clamp(min=1e-30)).max())
        return o, lse


EDGE = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_single_tokens_at_the_edges_of_tiles_and_pages(dtype, d, page):
    Setup4(EDGE, [1] * len(EDGE), d=d, page=page, dtype=dtype, behind=math.nan, seed=1).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h_kv,g", [(1, 1), (3, 2), (2, 8), (1, 16), (8, 4), (5, 1)])
def test_head_layouts(dtype, d, h_kv, g):
    Setup4([300, 41, 1000], [1, 3, 20], h_kv=h_kv, g=g, d=d, dtype=dtype, page=32, seed=2).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("news", [[7, 0, 33, 1, 130, 64], [1, 1, 0, 0, 0, 1], [0, 0, 0, 0, 700, 0]])
def test_chunks_of_every_length_beside_each_other(dtype, causal, news):
    Setup4([500, 20, 33, 1, max(131, news[4]), 64], news, dtype=dtype, page=16, spare=3, behind=math.nan, seed=3).check(causal)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_whole_prompts(dtype, d):
    Setup4([130, 257, 1], [130, 257, 1], d=d, dtype=dtype, page=64, seed=4).check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,page,h_kv,g", [(128, 16, 2, 4), (64, 16, 3, 2), (128, 64, 1, 16), (64, 256, 2, 8), (128, 32, 4, 1)])
@pytest.mark.parametrize("news", [[7, 0, 33, 1, 130, 64, 9], [40, 20, 0, 1, 0, 3, 0], [0, 0, 0, 0, 700, 0, 0]])
def test_chunks_in_wide_tables(causal, d, page, h_kv, g, news):
    Setup4([500, 20, 333, 1, max(131, news[4]), 64, 1500], news, h_kv=h_kv, g=g, d=d, page=page, width=3000 // page, behind=math.nan, seed=5).check(causal)


@pytest.mark.parametrize("lens,news,h_kv,g,d,page", [([6400], [380], 2, 4, 128, 64), ([6300], [600], 2, 4, 64, 16), ([6400, 70, 6000], [250, 1, 129], 2, 4, 128, 32),
                                                     ([6400], [380], 128, 1, 64, 16), ([9000, 70], [300, 1], 8, 4, 128, 16)])
def test_long_pieces(lens, news, h_kv, g, d, page):
    Setup4(lens, news, h_kv=h_kv, g=g, d=d, page=page, behind=math.nan, seed=6).check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_that_see_nothing(dtype):
    """Empty sequences with new rows, and more new rows than tokens: zeros and -inf."""
    s = Setup4([0, 3, 40], [2, 5, 41], dtype=dtype, spare=1, seed=7)
    o, lse = s.check()
    assert torch.isneginf(lse[:4]).all() and (o[:4] == 0).all() and torch.isneginf(lse[7]).all()
    s.check(causal=False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,news", [(5000, 1), (5000, 40), (20001, 2), (9000, 300)])
def test_long_caches_are_cut_and_joined(dtype, n, news):
    Setup4([n, 60], [news, 1], h_kv=1, g=4, dtype=dtype, page=64, seed=8).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h_kv,g,lens,news", [(1, 16, [17000, 30], [1, 1]), (1, 8, [8200, 9000, 50], [2, 1, 0]), (2, 16, [4100], [1]), (1, 1, [40000], [3])])
@pytest.mark.parametrize("d", [64, 128])
def test_long_caches_of_few_heads_are_joined_in_levels(dtype, h_kv, g, lens, news, d):
    Setup4(lens, news, h_kv=h_kv, g=g, d=d, dtype=dtype, page=64, seed=9).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("batch,new,h_kv,g", [(70, 1, 2, 4), (150, 2, 1, 2), (30, 20, 8, 1), (14, 30, 16, 4)])
def test_batches_of_many_sequences(dtype, batch, new, h_kv, g):
    lens = [(37 * i) % 400 + new for i in range(batch)]
    Setup4(lens, [new] * batch, h_kv=h_kv, g=g, d=64, dtype=dtype, page=32, seed=10).check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g,h_kv", [(1, 8), (2, 3), (4, 2), (8, 1)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("batch,many", [(12, 9), (40, 30), (70, 7)])
def test_tiles_of_few_rows(d, g, h_kv, causal, batch, many):
    """Few rows a sequence on the average: none, one or two, and many in one of them; lengths on both sides of 16, 32, 64 and 128 keys."""
    around = [16, 17, 31, 33, 47, 64, 65, 80, 96, 97, 127, 129, 200, 1100]
    lens = [around[i % len(around)] for i in range(batch)]
    news = [[0, 1, 0, 2, 0][i % 5] if g < 4 else [0, 1, 0, 1, 0][i % 5] for i in range(batch)]
    news[5 % batch] = 0
    news[5 % batch] = min(many, 8 * batch // g - sum(news) - 1)
    s = Setup4(lens, news, h_kv=h_kv, g=g, d=d, page=[16, 64][batch % 3 == 0], behind=math.nan, spare=1, seed=24)
    assert s.rows * g <= 8 * batch
    s.check(causal)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g,h_kv,lens,news", [(4, 8, [9000], [1]), (1, 2, [20000, 300], [3, 1]), (8, 1, [16000], [1]), (2, 4, [4000, 9001], [1, 2]), (4, 1, [33000, 5], [1, 1])])
def test_tiles_of_few_rows_are_cut_and_joined(d, g, h_kv, lens, news):
    Setup4(lens, news, h_kv=h_kv, g=g, d=d, page=64, behind=math.nan, seed=25).check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g,h_kv,m", [(1, 16, 33), (2, 8, 12), (4, 8, 9), (16, 8, 3)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("width,page", [(64, 16), (70, 64)])
def test_tiles_of_32_rows(d, g, h_kv, m, causal, width, page):
    """Between 16 and 80 rows a sequence on the average, in batches: tiles with one, one and a half and two groups of 16 rows; sequences without new tokens or shorter than
    them; lengths on both sides of 32, 64 and 128 keys, in caches that hold more and no more than a thousand."""
    around = [16, 700, 31, 33, 47, 64, 65, 5, 96, 97, 127, 129, 200, 1000, 0, 385]
    lens = [around[i % len(around)] for i in range(26)]
    news = [[m, m + 1, 0, 2 * m, 1, m // 2][i % 6] for i in range(26)]
    Setup4(lens, news, h_kv=h_kv, g=g, d=d, page=page, width=max(width * 16 // page, 1000 // page + 1), behind=math.nan, spare=2, seed=31).check(causal)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g,long,m", [(4, [9000, 1, 2500], 8), (4, [20000, 129, 128], 16), (8, [6001, 4097, 33], 5), (1, [12000, 7], 30)])
def test_tiles_of_32_rows_are_cut_and_joined(d, g, long, m):
    """A few long sequences beside short ones: some tiles are cut into many pieces, added up in one level and in two, and runs go over several tiles.  A block of V that is NaN
    late in the first sequence, and one of K in the second, are lost where they are seen and nowhere else."""
    h_kv, page = 8, 64
    lens = long + [200 + 17 * i for i in range(22)]
    news = [m, m - 1, 1][:len(long)] + [[m, m + 2, 0, 3][i % 4] for i in range(22)]
    news = [min(x, n) for x, n in zip(news, lens)]
    s = Setup4(lens, news, h_kv=h_kv, g=g, d=d, page=page, seed=32)
    clean, clean_lse = s.check()
    slots = [lens[0] - m // 2 - 1, max(lens[1] - 1, 0)]
    for b, tensor, head in ((0, 3, 1), (1, 1, 2)):
        s.codes[tensor][int(s.table[b, slots[b] // page]), head, slots[b] % page, d // 32 - 1] = 255
    s.place()
    o, lse = s.attend()
    lost = torch.zeros(o.shape, dtype=torch.bool)
    start = s.row_start.tolist()
    for b, head, span in ((0, 1, slice(d - 32, d)), (1, 2, slice(0, d))):
        for t in range(news[b]):
            lost[start[b] + t, head * g:(head + 1) * g, span] = lens[b] - news[b] + t >= slots[b]
    assert torch.equal(torch.isnan(o), lost)
    assert torch.equal(torch.isnan(lse[:start[1]]), torch.zeros_like(lse[:start[1]], dtype=torch.bool))
    assert torch.equal(torch.isnan(lse[start[1]:]), lost[start[1]:].any(-1))
    assert torch.equal(o[~lost], clean[~lost])


def test_tiles_of_32_rows_in_a_graph():
    """Replayed with other lengths, eager calls between: the flags of cut tiles are clear each time."""
    lens, news = [5000, 300, 2000] + [100] * 17, [8] * 20
    s = Setup4(lens, news, h_kv=8, g=4, page=64, seed=33)
    p, q = s.params(), s.q.to(DEV)
    ws = B.alloc_paged4_workspace(p, DEV)
    ws.zero_()
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dash_paged4_attend(p, s.gpu, q, s.start_gpu, o, ws, lse=lse)
    for other in (lens, [4999, 7, 0] + [33] * 17, [100] * 20, lens):
        s.gpu.lens.copy_(torch.tensor(other))
        want = s.attend()
        for _ in range(2):
            o.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g,h_kv", [(1, 2), (4, 8), (16, 1)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("batch,page", [(5, 16), (70, 64)])
def test_few_rows_beside_many(d, g, h_kv, causal, batch, page):
    """Sequences of up to 48 rows and of more have launches of their own: some of 48 and of one token more, prompts, none, and shorter ones than their new rows."""
    most = 48 // g
    kinds = [(700, most), (900, most + 1), (2100, 1100 // g + 900), (33, 1), (5, 9), (0, 2), (640, 0), (1500, most - 1), (20, 20), (257, 2 * most + 3)]
    seqs = [kinds[i % len(kinds)] for i in range(batch)]
    if batch > 10:
        seqs = [(n, min(m, 60)) for n, m in seqs[:-1]] + [(3000, 90 * batch // g)]
    s = Setup4([n for n, _ in seqs], [m for _, m in seqs], h_kv=h_kv, g=g, d=d, page=page, behind=math.nan, spare=1, seed=35, width=3200 // page)
    assert s.rows * g > 80 * batch
    s.check(causal)


def test_sequences_that_change_sides_in_a_graph():
    """Captured once; row starts and lengths are those of each replay."""
    s = Setup4([3000, 2000, 1000, 400], [200, 12, 13, 1], h_kv=8, g=4, page=64, seed=36)
    p, q = s.params(), s.q.to(DEV)
    ws = B.alloc_paged4_workspace(p, DEV)
    ws.zero_()
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dash_paged4_attend(p, s.gpu, q, s.start_gpu, o, ws, lse=lse)
    for start, lens in (([0, 200, 212, 225, 226], [3000, 2000, 1000, 400]), ([0, 5, 218, 219, 226], [3000, 1999, 1000, 390]), ([0, 12, 24, 36, 48], [2999, 2000, 30, 400]),
                        ([0, 56, 112, 168, 226], [3000, 2000, 1000, 57]), ([0, 226, 226, 226, 226], [3000, 1, 2, 3]), ([0, 200, 212, 225, 226], [3000, 2000, 1000, 400])):
        s.start_gpu.copy_(torch.tensor(start))
        s.gpu.lens.copy_(torch.tensor(lens))
        s.row_start, s.lens = torch.tensor(start, dtype=torch.int32), torch.tensor(lens, dtype=torch.int32)
        s.ref = P.Cache(s.ref.k, s.ref.v, s.table, s.lens)
        s.check()
        want = s.attend()
        for _ in range(2):
            o.fill_(77)
            lse.fill_(77)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_peaked_and_falling_logits(dtype):
    s = Setup4([700, 300], [3, 200], dtype=dtype, page=32, seed=11, qscale=30.0)
    s.check()
    kc, ks, vc, vs = s.codes
    s.codes[1] = torch.where(torch.arange(32)[None, None, :, None] < 16, ks, ks - 6)
    s.place()
    s.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strided_queries_outputs_and_pages(dtype):
    for layout in ("head", "token"):
        for news in ([1, 2], [70, 3]):
            s = Setup4([333, 90], news, dtype=dtype, page=32, layout=layout, seed=12)
            rows = s.q.shape[0]
            wide = torch.zeros((rows, 8, 3 * 128), dtype=dtype, device=DEV)
            q = wide[..., 128:256]
            q.copy_(s.q)
            s.check(q=q)
            by_head = torch.zeros((8, rows, 128), dtype=dtype, device=DEV).transpose(0, 1)
            by_head.copy_(s.q)
            s.check(q=by_head)


def test_a_given_scale():
    Setup4([300, 20], [2, 20], seed=13).check(scale=0.25)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_bad_page_spoils_its_own_sequence_only(dtype):
    """Table entries outside the pool take some page of it: nothing else changes."""
    s = Setup4([100, 100, 100], [1, 1, 1], dtype=dtype, page=16, seed=14)
    o, lse = s.check()
    for bad in (-1, 1 << 30, s.codes[0].shape[0]):
        s.gpu.table[1, 2] = bad
        o2, lse2 = s.attend()
        assert torch.equal(o2[[0, 2]], o[[0, 2]]) and torch.equal(lse2[[0, 2]], lse[[0, 2]])


def test_lengths_and_row_starts_out_of_range_are_clamped():
    s = Setup4([64, 64], [2, 2], page=16, seed=15)
    o, lse = s.check()
    s.gpu.lens[1] = 1 << 30                                      # the table's 64
    s.start_gpu[2] = 1 << 30                                     # the rows' 4
    o2, lse2 = s.attend()
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    s.gpu.lens[1], s.start_gpu[0] = -5, -7
    o2, lse2 = s.attend()
    assert torch.equal(o2[:2], o[:2]) and torch.isneginf(lse2[2:]).all() and (o2[2:] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("news", [[1], [3], [5], [40], [300]])
def test_a_block_that_is_nan_reaches_the_rows_that_see_its_token(dtype, d, news):
    """In V it spoils its 32 numbers of their outputs, in K their rows."""
    n, page, h_kv, g = 400, 16, 2, 4
    for tensor in (1, 3):
        s = Setup4([n, 60], [news[0], 1], h_kv=h_kv, g=g, d=d, page=page, dtype=dtype, seed=16)
        clean, clean_lse = s.check()
        slot, block = n - news[0] // 2 - 1, d // 32 - 1
        pg = int(s.table[0, slot // page])
        s.codes[tensor][pg, 1, slot % page, block] = 255
        s.place()
        o, lse = s.attend()
        sees = torch.arange(news[0]) + n - news[0] >= slot       # new tokens
        lost = torch.zeros(o.shape, dtype=torch.bool)
        rows = torch.nonzero(sees)[:, 0]
        span = slice(0, d) if tensor == 1 else slice(32 * block, 32 * block + 32)
        lost[rows, g:, span] = True
        assert torch.equal(torch.isnan(o), lost)
        assert torch.equal(torch.isnan(lse), lost.any(-1) if tensor == 1 else torch.zeros_like(lse, dtype=torch.bool))
        assert torch.equal(o[~lost], clean[~lost])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_query_that_is_nan_spoils_its_own_row(dtype):
    s = Setup4([100, 300], [3, 70], dtype=dtype, seed=17)
    clean, clean_lse = s.check()
    s.q[5, 3, 17] = math.nan
    o, lse = s.attend()
    lost = torch.zeros(lse.shape, dtype=torch.bool)
    lost[5, 3] = True
    assert torch.equal(torch.isnan(lse), lost) and torch.isnan(o[5, 3]).all()
    assert torch.equal(o[~lost], clean[~lost]) and torch.equal(lse[~lost], clean_lse[~lost])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_before_the_first_sequence(dtype):
    for news in ([2, 1], [90, 3]):
        s = Setup4([200, 100], news, dtype=dtype, seed=18)
        s.check()
        q = torch.cat((torch.full_like(s.q[:3], math.nan), s.q))
        s.start_gpu += 3
        s.q = q
        o2, lse2 = s.attend()
        want, wl, tol, ltol = P.attend(s.ref, q[3:], s.row_start, s.h_kv)
        assert ((o2[3:].double() - want).abs() <= tol).all() and ((lse2[3:].double() - wl).abs() <= ltol).all()
        assert (o2[:3] == 77).all() and (lse2[:3] == 77).all()


def test_pages_past_four_gigabytes():
    """Codes far behind the 32-bit offsets' end."""
    n_pages, page, h_kv, d = 1200, 1024, 32, 128                  # 2.5 GB of codes each
    gen = torch.Generator().manual_seed(19)
    c = B.PagedCache4.allocate(2, h_kv, 2 * n_pages, page, d, 2, DEV)
    pages = torch.tensor([[2 * n_pages - 1, 2 * n_pages - 2], [0, 2 * n_pages - 3]], dtype=torch.int32)
    c.table.copy_(pages)
    c.lens.copy_(torch.tensor([1500, 1100]))
    k, v = (torch.randn((4, h_kv, page, d), generator=gen) for _ in range(2))
    which = pages.reshape(-1).long()
    small = []
    for x, codes, scales in ((k, c.k_codes, c.k_scales), (v, c.v_codes, c.v_scales)):
        a, b = R.quantise(x)
        codes[which.to(DEV)], scales[which.to(DEV)] = a.to(DEV), b.to(DEV)
        small.append(R.values(a, b).float())
    q = torch.randn((2, h_kv, d), generator=gen).to(BF)
    start = torch.tensor([0, 1, 2], dtype=torch.int32)
    p = B.make_paged4_params(c, 2, h_kv)
    o, lse = torch.empty_like(q, device=DEV), torch.empty((2, h_kv), device=DEV)
    B.dash_paged4_attend(p, c, q.to(DEV), start.to(DEV), o, B.alloc_paged4_workspace(p, DEV), lse=lse)
    ref = P.Cache(*small, torch.tensor([[0, 1], [2, 3]], dtype=torch.int32), torch.tensor([1500, 1100], dtype=torch.int32))
    want, wl, tol, ltol = P.attend(ref, q, start, h_kv)
    assert ((o.cpu().double() - want).abs() <= tol).all() and ((lse.cpu().double() - wl).abs() <= ltol).all()
    # the last token of the first sequence anew, with another scale
    new = 100.0 * torch.randn((1, h_kv, d), generator=gen).to(BF)
    c.table[1] = -1
    B.dash_paged4_append(B.make_paged4_params(c, 1, h_kv), c, new.to(DEV), new.to(DEV), torch.tensor([0, 1, 1], dtype=torch.int32, device=DEV))
    pg, off = int(pages[0, 1]), 1499 % page
    for codes, scales in ((c.k_codes, c.k_scales), (c.v_codes, c.v_scales)):
        assert torch.equal(R.values(codes[pg, :, off].cpu(), scales[pg, :, off].cpu()), held(new[0]))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_two_captured_graphs_and_eager_calls_between_them(dtype):
    """Each graph has a workspace of its own; lengths change between replays."""
    s = Setup4([3000, 700, 40], [1, 1, 1], h_kv=1, g=8, dtype=dtype, page=64, seed=20, width=48)
    p, q = s.params(), s.q.to(DEV)
    runs = []
    for _ in range(2):
        ws = B.alloc_paged4_workspace(p, DEV)
        ws.zero_()
        o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.dash_paged4_attend(p, s.gpu, q, s.start_gpu, o, ws, lse=lse)
        runs.append((graph, o, lse, ws))                         # a graph's workspace lives as long as it
    for lens in ([3000, 700, 40], [2999, 1, 0], [5, 700, 33], [3000, 700, 40]):
        s.gpu.lens.copy_(torch.tensor(lens))
        want = s.attend()
        streams = [torch.cuda.Stream() for _ in runs]
        for st, (graph, o, lse, _) in zip(streams, runs):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                o.zero_()
                graph.replay()
        torch.cuda.synchronize()
        for _, o, lse, _ in runs:
            assert torch.equal(o.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])


def test_the_same_bits_every_time():
    for news in ([1, 1, 1], [200, 1, 3]):
        s = Setup4([5000, 3000, 100], news, h_kv=2, g=4, page=64, seed=22)
        first = s.attend()
        for _ in range(5):
            again = s.attend()
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ---- all of it, as it is used ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("graph", [False, True])
def test_prompts_and_steps(dtype, graph):
    """Two sequences: a prompt in two pieces beside one that decodes, then steps of both (captured once where `graph`).  Every call against the
    definitions, over the values that the cache holds."""
    h_q, h_kv, d, page = 8, 2, 128, 16
    rand = draws(23)
    r = B.make_rotary(d, DEV, scaling="linear", factor=2.0)
    theta = [t / 2 for t in R.thetas(d)]
    c = B.PagedCache4.allocate(2, h_kv, 40, page, d, 16, DEV)
    order = torch.randperm(40, generator=torch.Generator().manual_seed(1))[:32].view(2, 16)
    c.table.copy_(order)
    k_ref, v_ref = torch.zeros((40, h_kv, page, d)), torch.zeros((40, h_kv, page, d))
    lens = [0, 0]
    recorded = {}
    for news in ([50, 1], [37, 1], [1, 1], [1, 1], [1, 1]):
        rows = sum(news)
        q, k, v = rand(rows, h_q, d).to(dtype), rand(rows, h_kv, d).to(dtype), rand(rows, h_kv, d).to(dtype)
        lens = [a + b for a, b in zip(lens, news)]
        start = torch.tensor([0, news[0], rows], dtype=torch.int32)
        if graph and tuple(news) in recorded:
            g, qg, kg, vg, q_out, o, lse, sg = recorded[tuple(news)]
            qg.copy_(q), kg.copy_(k), vg.copy_(v)
            c.lens.copy_(torch.tensor(lens))
            g.replay()
        else:
            qg, kg, vg, sg = q.to(DEV), k.to(DEV), v.to(DEV), start.to(DEV)
            q_out, o, lse = torch.empty_like(qg), torch.empty_like(qg), torch.empty((rows, h_q), device=DEV)
            p = B.make_paged4_params(c, rows, h_q, dtype=dtype)
            ws = B.alloc_paged4_workspace(p, DEV)
            ws.zero_()
            def step():
                B.dash_paged4_append(p, c, kg, vg, sg, rotary=r, q=qg, q_out=q_out)
                B.dash_paged4_attend(p, c, q_out, sg, o, ws, lse=lse)
            c.lens.copy_(torch.tensor(lens))
            if graph and rows == 2:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    step()
                recorded[tuple(news)] = (g, qg, kg, vg, q_out, o, lse, sg)
                recorded["ws"] = ws
                g.replay()
            else:
                step()
        torch.cuda.synchronize()
        at = torch.tensor([x[3] for x in R.positions(lens, start)])
        check(q_out, q, at[:, None], theta, "halves")
        for row, b, slot, position in R.positions(lens, start):
            k_ref[order[b, slot // page], :, slot % page] = held(R.turn(k[row], torch.tensor(position), theta, "halves")[0]).float()
            v_ref[order[b, slot // page], :, slot % page] = held(v[row]).float()
        ref = P.Cache(k_ref, v_ref, order.to(torch.int32), torch.tensor(lens, dtype=torch.int32))
        want, wl, tol, ltol = P.attend(ref, q_out.cpu(), start, h_kv)
        assert ((o.cpu().double() - want).abs() <= tol).all() and ((lse.cpu().double() - wl).abs() <= ltol).all()
    # handed over to a cache of whole numbers: the same attention
    kp, vp = (torch.empty((40, h_kv, page, d), dtype=dtype, device=DEV) for _ in range(2))
    B.dash_paged4_unpack(p, c, kp, vp)
    assert torch.equal(kp.cpu().float()[order.reshape(-1)], k_ref[order.reshape(-1)])
    full = B.PagedCache(kp, vp, c.table, c.lens)
    fp = B.make_paged_params(full, 2, h_q)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    B.dash_paged_attend(fp, full, q_out, sg, o2, B.alloc_paged_workspace(fp, DEV), lse=lse2)
    assert ((o2.cpu().double() - want).abs() <= tol).all() and ((lse2 - lse).abs().cpu() <= 2 * ltol).all()
