"""CPU-side tests of rotary positions and of the paged cache in 4 bits: the table of turns, refusals before any launch, the binding's checks, and the
plain forms of the GPU tests."""
import ctypes
import dataclasses
import decimal
import math
import os
import shutil
import subprocess

import pytest
import torch

import paged4_ref as R
from test_library_paged import params
from paper_2605_18753_amd import binding as B

TURN = 1 << 64


def turns(rot, freq=None, scaling=0, base=10000.0, factor=1.0, original=0.0, low=0.0, high=0.0, out=True):
    x = torch.zeros(64, dtype=torch.int64)
    f = None if freq is None else torch.tensor(freq, dtype=torch.float64)
    rc = B.load_library().dash_rotary_turns(rot, None if f is None else f.data_ptr(), scaling, base, factor, original, low, high, x.data_ptr() if out else None)
    return rc, [int(t) % TURN for t in x[:rot // 2]]


@pytest.mark.parametrize("rot", [16, 48, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 10.0])
def test_turns_are_the_thetas_as_fractions(rot, base):
    """long double holds a theta to 64 bits; its power and the division are off by a few units."""
    rc, got = turns(rot, base=base)
    assert rc == 0
    for t, g in zip(R.thetas(rot, base), got):
        want = t / R.TWO_PI * TURN
        assert abs(want - g) <= 1 + abs(want) * decimal.Decimal(2) ** -60


@pytest.mark.parametrize("scaling,kw", [(1, dict(factor=4.0)), (2, dict(factor=8.0)), (3, dict(factor=16.0, original=8192.0, low=1.0, high=32.0))])
def test_scaled_turns(scaling, kw):
    rc, got = turns(64, scaling=scaling, **kw)
    assert rc == 0
    D = decimal.Decimal
    f, theta = D(kw["factor"]), R.thetas(64)
    if scaling == 1:
        want = [t / f for t in theta]
    elif scaling == 2:
        want = [(D(10000).ln() * -2 * i / 64 + f.ln() * 64 / 62 * -2 * i / 64).exp() for i in range(32)]
        assert abs(want[-1] * f / theta[-1] - 1) < D("1e-30") and want[0] == 1   # the slowest divided by the factor, the fastest kept
    else:
        want = []
        for t in theta:
            c = min(max((D(8192) * t / R.TWO_PI - 1) / 31, D(0)), D(1))
            want.append(t * (c + (1 - c) / f))
        assert want[0] == theta[0] and want[-1] == theta[-1] / f
    for t, g in zip(want, got):
        assert abs(t / R.TWO_PI * TURN - g) <= 1 + t / R.TWO_PI * TURN * D(2) ** -58


def test_frequencies_of_the_callers_own():
    freq = [1.0, -1.0, 0.0, 100.0, -0.001, 2 * math.pi, 1e-30, 3.0]
    rc, got = turns(16, freq=freq, base=-5.0, scaling=77)        # what follows the frequencies is not used
    assert rc == 0 and (got[0] + got[1]) % TURN == 0 and got[2] == 0 and got[6] == 0
    for f, g in zip(freq, got):
        want = decimal.Decimal(f) / R.TWO_PI % 1 * TURN
        far = (want - g) % TURN
        assert min(far, TURN - far) <= 1 + abs(decimal.Decimal(f) / R.TWO_PI) * TURN * decimal.Decimal(2) ** -62


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(rot=64, base=0.0), dict(rot=64, base=math.nan), dict(rot=64, base=math.inf),
                                dict(rot=64, scaling=4), dict(rot=64, scaling=-1), dict(rot=64, scaling=1, factor=0.0), dict(rot=64, scaling=2, factor=-1.0),
                                dict(rot=64, scaling=3, factor=2.0), dict(rot=64, scaling=3, factor=2.0, original=100.0, low=2.0, high=2.0),
                                dict(rot=16, freq=[math.nan] * 8), dict(rot=16, freq=[math.inf] * 8), dict(rot=64, out=False)])
def test_turns_refuse(kw):
    rc, got = turns(**kw)
    assert rc == -1 and not any(got)


# ---- refusals of the C ABI -------------------------------------------------------------------------------------------
def plan(**kw):
    r = B.dash_rotary_plan(64, 0, 1.0, 0, 256)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def rparams(**kw):
    p = B.dash_rotary_params()
    base = dict(batch=2, h_q=4, h_kv=2, n_q=10, n_kv=10, head_dim=128, dtype=B.DASH_BF16)
    base.update({k: v for k, v in kw.items() if not k.endswith("stride") or k == "pos_stride"})
    for k, v in base.items():
        setattr(p, k, v)
    for k in ("q_stride", "q_out_stride", "k_stride", "k_out_stride"):
        getattr(p, k)[:] = kw.get(k, [10 * 4 * 128, 10 * 128, 128])
    return p


def apply(p=None, r=None, q=256, q_out=256, k=512, k_out=512):
    return B.load_library().dash_rotary_apply(rparams() if p is None else p, plan() if r is None else r, None, q, q_out, k, k_out, None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -1), (dict(h_q=0), -1), (dict(h_kv=0), -1), (dict(n_q=0), -1), (dict(n_kv=-1), -1), (dict(n_q=11), -1), (dict(head_dim=0), -1), (dict(dtype=2), -1),
    (dict(inverse=2), -1), (dict(reserved=1), -1), (dict(pos_stride=-1), -1), (dict(q_stride=[-8, 8, 8]), -1), (dict(k_out_stride=[8, 4, 8]), -1),
    (dict(q_out_stride=[10 * 4 * 128, 10 * 128, 136]), -1), (dict(head_dim=96), -2), (dict(batch=1 << 30), -2), (dict(h_q=1 << 16), -2)])
def test_rotary_refuses_parameters(kw, code):
    assert apply(rparams(**kw)) == code


def test_rotary_refuses_pointers():
    for kw in (dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(q=264, q_out=264), dict(k=520, k_out=520), dict(q=None, q_out=None, k=None, k_out=None)):
        assert apply(**kw) == -1, kw
    assert B.load_library().dash_rotary_apply(None, plan(), None, 256, 256, None, None, None) == -1
    assert B.load_library().dash_rotary_apply(rparams(), None, None, 256, 256, None, None, None) == -1


PLANS = [(dict(turns=None), -1), (dict(turns=260), -1), (dict(reserved=1), -1), (dict(layout=2), -1), (dict(rot_dim=0), -1), (dict(rot_dim=144), -1), (dict(mscale=0.0), -1),
         (dict(mscale=-1.0), -1), (dict(mscale=math.nan), -1), (dict(mscale=math.inf), -1), (dict(rot_dim=24), -2), (dict(rot_dim=2), -2)]


def params4(**kw):
    d = kw.get("head_dim", 128)
    base = dict(k_stride=[2 * 64 * d // 2, 64 * d // 2, d // 2], v_stride=[2 * 64 * d // 2, 64 * d // 2, d // 2])
    base.update(kw)
    return params(**base)


def call4(name, p, r=None, ws=4096, n=1 << 40, **kw):
    """The entry point with pointers that no launch may reach (the refusals come first)."""
    a = dict(k_new=256, v_new=256, q=None, q_out=None, k=256, v=256, ks=256, vs=256, o=256, lse=256, row_start=256, lens=256, table=256, seen=256, weights=None, pos=None)
    if name == "attend":
        a["q"] = 256
    a.update(kw)
    lib, g = B.load_library(), a.get
    p = ctypes.byref(p)
    if name == "rotary":
        return lib.dash_paged_append_rotary(p, r, g("q"), g("q_out"), g("k_new"), g("v_new"), g("k"), g("v"), g("row_start"), g("lens"), g("table"), g("weights"), g("pos"),
                                            g("seen"), None)
    if name == "append":
        return lib.dash_paged4_append(p, r, g("q"), g("q_out"), g("k_new"), g("v_new"), g("k"), g("ks"), g("v"), g("vs"), g("row_start"), g("lens"), g("table"), g("seen"), None)
    if name == "attend":
        return lib.dash_paged4_attend(p, g("q"), g("k"), g("ks"), g("v"), g("vs"), g("row_start"), g("lens"), g("table"), g("o"), g("lse"), ws, n, None)
    return lib.dash_paged4_unpack(p, g("k"), g("ks"), g("v"), g("vs"), g("k_out", 256), g("v_out", 256), None)


@pytest.mark.parametrize("kw,code", PLANS)
def test_plans_that_every_call_refuses(kw, code):
    assert apply(r=plan(**kw)) == code
    assert call4("rotary", params(), plan(**kw)) == code
    assert call4("append", params4(), plan(**kw)) == code
    if "rot_dim" not in kw:
        assert call4("rotary", params(head_dim=64), plan(**{**kw, "rot_dim": 64})) == code
    assert call4("rotary", params(head_dim=64), plan(rot_dim=80)) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -1), (dict(h_q=7), -1), (dict(h_kv=0), -1), (dict(dtype=2), -1), (dict(causal=2), -1), (dict(n_pages=0), -1),
    (dict(max_pages=0), -1), (dict(page_size=0), -1), (dict(reserved=1), -1), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1),
    (dict(k_stride=[8192, 4096, 48]), -1), (dict(v_stride=[8192, 4096, 72]), -1), (dict(k_stride=[-16, 4096, 64]), -1), (dict(v_stride=[8192, 4104, 64]), -1),
    (dict(head_dim=96), -2), (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=2048), -2),
    (dict(h_q=64, h_kv=2), -2), (dict(h_q=6, h_kv=2), -2), (dict(max_pages=1 << 20), -2), (dict(k_stride=[8192, 4096, 1 << 26]), -2),
    (dict(v_stride=[8192, 4096, 1 << 62]), -2), (dict(batch=1 << 20), -2)])
def test_parameters_that_every_call_refuses(kw, code):
    for name in ("append", "attend", "unpack"):
        assert call4(name, params4(**kw)) == code, name
    n = ctypes.c_size_t(0)
    f = B.load_library().dash_paged4_workspace_bytes
    assert f(ctypes.byref(params4(**kw)), ctypes.byref(n)) == code
    assert f(ctypes.byref(params4()), None) == -1 and f(None, ctypes.byref(n)) == -1


def test_parameters_of_the_packed_rows():
    for name in ("append", "attend"):
        assert call4(name, params4(n_rows=0)) == -1 and call4(name, params4(n_rows=(1 << 28) + 1)) == -2
    for s in ("q_stride", "o_stride"):
        for bad in ([1024, 4], [-8, 128]):
            assert call4("attend", params4(**{s: bad})) == -1
            assert call4("append", params4(**{s: bad}), plan(), q=256, q_out=512) == -1
            assert call4("rotary", params(**{s: bad}), plan(), q=256, q_out=512) == -1
    for name in ("append", "rotary"):
        base = params4 if name == "append" else params
        assert call4(name, base(k_new_stride=[4, 128]), plan()) == -1 and call4(name, base(v_new_stride=[256, -8]), plan()) == -1
        assert call4(name, base(q_stride=[2048, 128]), plan(), q=256, q_out=256) == -1           # in place with other strides
        assert call4(name, base(), plan(), q=256) == -1 and call4(name, base(), plan(), q_out=256) == -1
    assert call4("append", params4(), None, q=256, q_out=512) == -1                              # queries without a plan


@pytest.mark.parametrize("name", ["rotary", "append"])
def test_queries_are_not_written_over_what_is_read(name):
    """16 rows of two heads of 128 in bf16 with strides of 256 and 128 elements: 8192 bytes.  Fused rows: 6 heads, q the first two."""
    p = params(n_rows=16, h_q=2, h_kv=2) if name == "rotary" else params4(n_rows=16, h_q=2, h_kv=2)
    far = 1 << 20
    assert (p.q_stride[0], p.q_stride[1], p.k_new_stride[0]) == (256, 128, 256)
    for kw in (dict(q=far, q_out=far + 16), dict(q=far + 8176, q_out=far), dict(q=far, q_out=4 * far, k_new=4 * far), dict(q=far, q_out=4 * far, v_new=4 * far + 8176),
               dict(q=far, q_out=far, k_new=far + 256), dict(q=far, q_out=4 * far + 256, v_new=4 * far)):
        a = dict(k_new=2 * far, v_new=3 * far)
        a.update(kw)
        assert call4(name, p, plan(), **a) == -1, kw
    for x in (p.q_stride, p.o_stride, p.k_new_stride, p.v_new_stride):
        x[0] = 768
    for kw in (dict(k_new=far + 384), dict(v_new=far + 256), dict(q_out=far + 128), dict(k_new=far + 1536 - 256), dict(k_new=far + 1536 + 256)):
        a = dict(q=far, q_out=far, k_new=far + 512, v_new=far + 1024)
        a.update(kw)
        assert call4(name, p, plan(), **a) == -1, kw
    for x in (p.q_stride, p.o_stride, p.k_new_stride, p.v_new_stride):                           # rows of heads of (q, k, v)
        x[1] = 384
    for kw in (dict(k_new=far + 128), dict(v_new=far + 640), dict(k_new=far + 768 + 16)):
        a = dict(q=far, q_out=far, k_new=far + 256, v_new=far + 512)
        a.update(kw)
        assert call4(name, p, plan(), **a) == -1, kw


@pytest.mark.parametrize("name,needed", [
    ("rotary", ("k_new", "v_new", "k", "v", "row_start", "lens", "table")), ("append", ("k_new", "v_new", "k", "v", "ks", "vs", "row_start", "lens", "table")),
    ("attend", ("q", "k", "v", "ks", "vs", "row_start", "lens", "table", "o")), ("unpack", ("k", "v", "ks", "vs", "k_out", "v_out"))])
def test_null_and_misaligned_pointers(name, needed):
    p = params() if name == "rotary" else params4()
    for x in needed:
        assert call4(name, p, plan(), **{x: None}) == -1, x
    for x in set(needed) & {"k_new", "v_new", "q", "k", "v", "ks", "vs", "o", "k_out", "v_out"}:
        assert call4(name, p, plan(), **{x: 264}) == -1, x


def test_workspaces():
    n = ctypes.c_size_t(0)
    f = B.load_library().dash_paged4_workspace_bytes
    assert f(ctypes.byref(params4()), ctypes.byref(n)) == 0
    for kw in (dict(ws=None), dict(ws=4097), dict(n=0), dict(n=n.value - 1)):
        assert call4("attend", params4(), **kw) == -3, kw
    one = n.value
    for rows in (1, 64, 5000, 1 << 20):                          # one workspace serves every number of rows
        assert f(ctypes.byref(params4(n_rows=rows)), ctypes.byref(n)) == 0 and n.value == one
    # fp32: 512 threads for 16 rows of a kv-head's group, fewer than 2^32
    for rows, batch, h, code in ((1 << 28, 1, 1, -2), ((((1 << 23) - 1) << 4) - 1, 1, 1, -3)):
        assert call4("attend", params4(n_rows=rows, batch=batch, h_q=h, h_kv=h, head_dim=64, dtype=B.DASH_F32), n=0) == code


# ---- the binding -----------------------------------------------------------------------------------------------------
def test_make_rotary_refuses():
    for kw in (dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=160), dict(rot_dim=1 << 40), dict(layout="pairs"), dict(scaling="more"), dict(scaling="linear", factor=0.0),
               dict(base=-1.0), dict(frequencies=[1.0] * 31), dict(frequencies=[math.nan] * 32)):
        with pytest.raises(B.DashError):
            B.make_rotary(**{**dict(rot_dim=64, device="cpu"), **kw})
    r = B.make_rotary(64, "cpu", layout="adjacent", mscale=1.5)
    assert (r.plan.rot_dim, r.plan.layout, r.plan.mscale, r.plan.turns) == (64, 1, 1.5, r.turns.data_ptr())


def test_rotary_binding_refuses_tensors_that_do_not_fit():
    r = B.make_rotary(64, "cpu")
    q, k = torch.zeros((2, 4, 10, 64)), torch.zeros((2, 2, 10, 64))
    good = dict(q=q, q_out=q.clone(), k=k, k_out=k.clone(), pos=torch.zeros((2, 10), dtype=torch.int32))
    def run(**kw):
        a = {**good, **kw}
        B.dash_rotary(r, a["q"], a["q_out"], a["k"], a["k_out"], pos=a["pos"], start=a.get("start", 0))
    wide = torch.zeros((2, 4, 10, 128))
    fused = torch.zeros((2, 10, 6, 64))
    for kw in (dict(q=None), dict(k_out=None), dict(q=q[0]), dict(q_out=q.clone()[:, :2]), dict(q_out=q.bfloat16()), dict(q=q.half(), q_out=q.half()), dict(k=k.bfloat16(), k_out=k.bfloat16()),
               dict(q=wide[..., ::2], q_out=wide[..., ::2]), dict(k=k[:1], k_out=k[:1].clone()), dict(q=q[..., :32], q_out=q[..., :32]), dict(q=q[:, :, :0], q_out=q[:, :, :0]),
               dict(q_out=q[:, :1].expand(-1, 4, -1, -1)), dict(q=wide[..., :64], q_out=wide[..., 32:96]), dict(q=wide[..., :64], q_out=wide[:, :, :, 16:80]),
               dict(pos=torch.zeros(9, dtype=torch.int32)), dict(pos=torch.zeros(10, dtype=torch.int64)), dict(pos=torch.zeros((10, 2), dtype=torch.int32).t()), dict(pos=torch.zeros((1, 10), dtype=torch.int32)),
               dict(start=1 << 31), dict(k_out=good["q_out"][:, :2]), dict(q=None, q_out=None, k=None, k_out=None),
               dict(q=fused[:, :, :4].transpose(1, 2), q_out=fused[:, :, :4].transpose(1, 2), k=fused[:, :, 3:5].transpose(1, 2), k_out=fused[:, :, 3:5].transpose(1, 2))):
        with pytest.raises(B.DashError) as e:
            run(**kw)
        assert "GPU" not in str(e.value), kw
    ok = [dict(), dict(q=None, q_out=None), dict(k=None, k_out=None), dict(q_out=q, k_out=k), dict(pos=None), dict(pos=torch.zeros(10, dtype=torch.int32)),
          dict(q=fused[:, :, :4].transpose(1, 2), q_out=fused[:, :, :4].transpose(1, 2), k=fused[:, :, 4:].transpose(1, 2), k_out=fused[:, :, 4:].transpose(1, 2))]
    each = torch.zeros((2, 10, 4, 3, 64))                        # (q, k, v) of each head side by side
    qe, ke = each[..., 0, :].transpose(1, 2), each[..., 1, :].transpose(1, 2)
    ok.append(dict(q=qe, q_out=qe, k=ke, k_out=ke))
    half = each.view(2, 10, 4, 192)[..., 32:96].transpose(1, 2)
    with pytest.raises(B.DashError, match="overlap"):
        run(q=qe, q_out=qe, k=half, k_out=half)
    for kw in ok:
        with pytest.raises(B.DashError, match="GPU"):            # nothing wrong but where the tensors lie
            run(**kw)
    r.turns = r.turns.clone()
    with pytest.raises(B.DashError, match="table"):
        run()


def cache4(batch=2, h_kv=2, n_pages=8, page=16, d=64):
    return B.PagedCache4.allocate(batch, h_kv, n_pages, page, d, 4, "cpu")


def test_paged4_binding_refuses_tensors_that_do_not_fit():
    c = cache4()
    p = B.make_paged4_params(c, 3, 4)
    assert (p.batch, p.h_kv, p.h_q, p.page_size, p.n_pages, p.max_pages, p.head_dim, p.n_rows, p.dtype) == (2, 2, 4, 16, 8, 4, 64, 3, B.DASH_BF16)
    assert list(p.k_stride) == [2 * 16 * 32, 16 * 32, 32] and (c.table == -1).all()
    ws, start, r = torch.empty(1 << 20, dtype=torch.uint8), torch.zeros(3, dtype=torch.int32), B.make_rotary(64, "cpu")
    q, kn, lse = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.zeros((3, 4))
    attend = lambda c=c, p=p, q=q, o=q.clone(), s=start, lse=lse: B.dash_paged4_attend(p, c, q, s, o, ws, lse=lse)  # noqa: E731
    append = lambda c=c, p=p, k=kn, v=kn, s=start, **kw: B.dash_paged4_append(p, c, k, v, s, **kw)  # noqa: E731
    pages = torch.zeros((8, 2, 16, 64), dtype=torch.bfloat16)
    unpack = lambda c=c, p=p, k=pages, v=pages.clone(): B.dash_paged4_unpack(p, c, k, v)  # noqa: E731
    for f in (attend, append, unpack, lambda: append(rotary=r), lambda: append(rotary=r, q=q, q_out=q), lambda: append(rotary=r, q=q, q_out=q.clone())):
        with pytest.raises(B.DashError, match="GPU"):            # nothing wrong but where the tensors lie
            f()
    bad = [lambda: attend(q=q[:2]), lambda: attend(q=q.float()), lambda: attend(o=q[:, :3]), lambda: attend(s=start.long()), lambda: attend(lse=lse.t()),
           lambda: append(k=kn[:2]), lambda: append(v=kn.float()), lambda: append(q=q, q_out=q), lambda: append(rotary=r, q=q), lambda: append(rotary=r, q_out=q),
           lambda: append(rotary=r, q=q, q_out=q[:, :2]), lambda: append(rotary=r, q=q[:, :, :32], q_out=q[:, :, :32]),
           lambda: append(rotary=r, q=torch.zeros((4, 4, 64), dtype=torch.bfloat16)[:3], q_out=q.float()), lambda: unpack(k=pages.float()), lambda: unpack(v=pages[:4]),
           lambda: unpack(k=pages.transpose(1, 2))]
    over = torch.zeros((4, 4, 64), dtype=torch.bfloat16)
    bad += [lambda: append(rotary=r, q=over[:3], q_out=over[1:])]
    for field, x in (("k_codes", c.k_codes[:4]), ("v_codes", c.v_codes.to(torch.int8)), ("k_codes", c.k_codes[..., ::2]), ("k_scales", c.k_scales[:4]), ("v_scales", c.v_scales.transpose(1, 2)),
                     ("k_scales", c.k_scales.to(torch.int8)), ("table", c.table.long()), ("lens", c.lens[:1]), ("lens", None), ("k_codes", c.k_codes[0])):
        other = dataclasses.replace(c, **{field: x})
        bad += [lambda o=other: attend(c=o), lambda o=other: append(c=o), lambda o=other: unpack(c=o), lambda o=other: B.make_paged4_params(o, 3, 4)]
    bad += [lambda: append(c=dataclasses.replace(c, seen=c.lens.long())), lambda: append(c=dataclasses.replace(c, seen=c.lens[:1]))]
    for other in (cache4(batch=3), cache4(h_kv=4), cache4(n_pages=9), cache4(page=32), cache4(d=128)):
        bad += [lambda o=other: attend(c=o), lambda o=other: append(c=o), lambda o=other: unpack(c=o)]
    bad += [lambda: B.make_paged4_params(c, 3, 4, dtype=torch.float16), lambda: B.make_paged4_params(c, 1 << 31, 4), lambda: attend(p=B.dash_paged_params(dtype=7))]
    for i, f in enumerate(bad):
        with pytest.raises(B.DashError) as e:
            f()
        assert "GPU" not in str(e.value), i
    full = B.PagedCache.allocate(2, 2, 8, 16, 64, 4, "cpu")
    fp = B.make_paged_params(full, 3, 4)
    for kw in (dict(q=q), dict(q=q, q_out=q[:2]), dict(q=q.float(), q_out=q.float())):
        with pytest.raises(B.DashError) as e:
            B.dash_paged_append_rotary(fp, full, r, kn, kn, start, **kw)
        assert "GPU" not in str(e.value)
    with pytest.raises(B.DashError, match="GPU"):
        B.dash_paged_append_rotary(fp, full, r, kn, kn, start, q=q, q_out=q)


# ---- the plain forms -------------------------------------------------------------------------------------------------
def test_the_plain_rotation():
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((3, 64), generator=gen, dtype=torch.float64)
    pos = torch.tensor([0, 3, 1000])
    for layout in ("halves", "adjacent"):
        y, tol = R.turn(x, pos, R.thetas(32), layout)
        assert torch.equal(y[0], x[0]) and torch.equal(y[:, 32:], x[:, 32:]) and (tol[:, :32] > 0).all()
        one, two = R.pairs_of(32, layout)
        z = torch.complex(x[..., one], x[..., two]) * torch.exp(1j * pos[:, None] * torch.tensor([float(t) for t in R.thetas(32)], dtype=torch.float64))
        assert (z.real - y[..., one]).abs().max() < 1e-12 and (z.imag - y[..., two]).abs().max() < 1e-12
        back, _ = R.turn(y, pos, R.thetas(32), layout, inverse=True)
        assert (back - x).abs().max() < 1e-14
        assert (R.turn(x, pos + 5, R.thetas(32), layout)[0] - R.turn(y, torch.tensor(5), R.thetas(32), layout)[0]).abs().max() < 1e-13
    assert abs(float(R.angles(torch.tensor([10 ** 9]), [1.0])[0, 0]) - math.remainder(10 ** 9, 2 * math.pi)) < 1e-6


def test_the_plain_quantisation():
    x = torch.zeros(5, 32, dtype=torch.float64)
    x[0, :8] = torch.tensor([6.0, 0.25, 0.75, 1.25, -1.75, 2.5, -3.5, 5.0])
    x[1, :3] = torch.tensor([7.25, 1.0, -0.3])
    x[2, :3] = torch.tensor([7.26, 1.0, -0.3])
    x[3, 5] = math.inf
    v = R.values(*R.quantise(x))
    assert v[0, :8].tolist() == [6, 0, 1, 1, -2, 2, -4, 4]        # ties to the even code
    assert v[1, :3].tolist() == [6, 1, -0.5] and v[2, :3].tolist() == [8, 1, 0] and torch.isnan(v[3]).all() and (v[4] == 0).all()
    gen = torch.Generator().manual_seed(2)
    y = torch.randn((4000, 32), generator=gen, dtype=torch.float64) * 2 ** torch.rand((4000, 1), generator=gen, dtype=torch.float64)
    held = R.values(*R.quantise(y))
    assert torch.equal(R.values(*R.quantise(held)), held)         # what is held is held as it is
    rms = float(((held - y) ** 2).mean().sqrt() / (y ** 2).mean().sqrt())
    assert 0.110 < rms < 0.114                                   # 0.112 by the figures that the border of 7.25 was chosen by
    codes, scales = R.quantise(y)
    unit = torch.exp2(scales.double() - 127)
    # no further off than half the step where it is: 0.25 below 2, 0.5 below 4, 1 below 6, and at the largest up to 1.25
    assert ((held - y).abs() <= torch.where(y.abs() < 2 * unit, 0.25, torch.where(y.abs() < 4 * unit, 0.5, 1.25)) * unit).all()


# ---- tensors in each other's span ------------------------------------------------------------------------------------
def elements(x):
    """The elements' places in their storage."""
    return torch.arange(x.untyped_storage().size() // x.element_size()).as_strided(x.shape, x.stride(), x.storage_offset())


def share(x, y):
    return x.untyped_storage().data_ptr() == y.untyped_storage().data_ptr() and bool(torch.isin(elements(x), elements(y)).any())


def spans(batch, h_q, h_kv, n, d, seed):
    """Queries and keys cut out of one tensor, its dimensions in any order, each at a place of its own."""
    gen = torch.Generator().manual_seed(seed)
    draw = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=gen))  # noqa: E731
    order = torch.randperm(3, generator=gen).tolist()            # which of batch, head and token lies outermost
    sizes = [batch, h_q + h_kv, n]
    room = [m + draw(0, 2) for m in sizes]
    x = torch.zeros([room[i] for i in order] + [d + 16 * draw(0, 1)])
    x = x.permute(*[order.index(i) for i in range(3)], 3)
    def part(heads):
        b, h, t = (draw(0, room[i] - m) for i, m in ((0, batch), (1, heads), (2, n)))
        return x[b:b + batch, h:h + heads, t:t + n, :d]
    return part(h_q), part(h_kv)


def test_tensors_that_share_elements_are_told_from_those_that_do_not():
    """In place on both: refused where they share elements, and nowhere else."""
    r = B.make_rotary(64, "cpu")
    said = {True: 0, False: 0}
    for seed in range(300):
        gen = torch.Generator().manual_seed(seed)
        batch, h_q, h_kv, n = (int(torch.randint(1, m, (1,), generator=gen)) for m in (4, 5, 3, 6))
        q, k = spans(batch, h_q, h_kv, n, 64, seed)
        with pytest.raises(B.DashError) as e:
            B.dash_rotary(r, q, q, k, k)
        said[share(q, k)] += 1
        assert ("overlap" if share(q, k) else "GPU") in str(e.value), (seed, q.shape, q.stride(), k.shape, k.stride(), k.storage_offset() - q.storage_offset())
    assert min(said.values()) > 50


def test_batches_inside_of_a_tokens_row():
    """[tokens, sequences, heads, d]: the queries' second sequence is the keys' first; heads of one tensor, and sequences in both, are apart."""
    r = B.make_rotary(64, "cpu")
    x = torch.zeros((10, 5, 6, 64))
    pairs = [(x[:, 0:4, :4].permute(1, 2, 0, 3), x[:, 1:5, :4].permute(1, 2, 0, 3), True), (x[:, 0:4, :4].permute(1, 2, 0, 3), x[:, 0:4, 4:].permute(1, 2, 0, 3), False),
             (x[:, 0:4, :4].permute(1, 2, 0, 3), x[:, 1:5, 4:].permute(1, 2, 0, 3), False), (x[:, 0:2, :4].permute(1, 2, 0, 3), x[:, 2:4, :4].permute(1, 2, 0, 3), False)]
    one = torch.zeros((10, 3, 64))
    pairs.append((one[:, 0:2].transpose(0, 1).unsqueeze(1), one[:, 1:3].transpose(0, 1).unsqueeze(1), True))
    for q, k, meet in pairs:
        assert share(q, k) == meet
        with pytest.raises(B.DashError, match="overlap" if meet else "GPU"):
            B.dash_rotary(r, q, q, k, k)


STRIDED = r"""
#include <cstdio>
#include <set>
#include <vector>
#include "strided.h"
using namespace dash;
static unsigned state = 1;
static int pick(int n) { state = state * 1664525u + 1013904223u; return (state >> 8) % n; }
template <typename F> static void each(const Strided& x, F f) {
  long n[3] = {1, 1, 1}, s[3] = {0, 0, 0};
  for (int i = 0; i < x.dims; i++) { n[i] = x.size[i]; s[i] = x.stride[i]; }
  for (int a = 0; a < n[0]; a++) for (int b = 0; b < n[1]; b++) for (int c = 0; c < n[2]; c++) f(a * s[0] + b * s[1] + c * s[2]);
}
// small tensors against the set of their elements; strides that often lie next to where a dimension ends
static Strided some(int d, int place) {
  Strided x = {(const void*)(long)(16 * place), 1 + pick(3), {}, {}};
  long inner = d;
  for (int i = 0; i < x.dims; i++) {
    x.size[i] = 1 + pick(4);
    x.stride[i] = pick(3) ? inner + pick(3) - 1 + d * pick(2) : pick(40);
    inner = x.stride[i] * (x.size[i] - 1) + inner;
  }
  if (pick(2) && x.dims > 1) { std::swap(x.size[0], x.size[1]); std::swap(x.stride[0], x.stride[1]); }
  return x;
}
int main() {
  int bad = 0, found[2] = {0, 0};
  for (int t = 0; t < 20000; t++) {
    const int d = 1 + pick(8);
    const Strided x = some(d, 0);
    std::set<long> on;
    bool repeats = false;
    each(x, [&](long at) { for (int e = 0; e < d; e++) repeats |= !on.insert(at + e).second; });
    found[repeats]++;
    bad += strided_repeats(x, d) != repeats;
  }
  // a torch layout of the largest sizes takes a few steps, whatever lies outermost
  const Strided wide = {nullptr, 3, {128, 1l << 40, 1l << 33}, {1 << 20, 65536, 128}};
  bad += strided_repeats(wide, 128) || strided_repeats({nullptr, 3, {1l << 62, 1l << 62, 128}, {2, 1, 5}}, 128);
  std::printf("%d wrong, %d apart, %d not\n", bad, found[0], found[1]);
  return bad != 0 || found[0] < 2000 || found[1] < 2000;
}
"""

MEET = STRIDED[:STRIDED.index("int main")] + r"""
int main() {
  int bad = 0, found[2] = {0, 0};
  for (int t = 0; t < 20000; t++) {
    const int d = 1 + pick(8);
    Strided x = some(d, 0), y = pick(2) ? some(d, 0) : x;
    y.at = (const void*)(long)(2 * pick(60));
    if (x.dims != y.dims) continue;
    if (pick(2)) std::swap(x, y);
    std::set<long> on;
    bool meet = false;
    const long off = ((long)y.at - (long)x.at) / 2;
    each(x, [&](long at) { for (int e = 0; e < d; e++) on.insert(at + e); });
    each(y, [&](long at) { for (int e = 0; e < d; e++) meet |= on.count(off + at + e) > 0; });
    found[meet]++;
    bad += strided_meet(x, y, d, 2) != meet;
  }
  std::printf("%d wrong, %d apart, %d not\n", bad, found[0], found[1]);
  return bad != 0 || found[0] < 2000 || found[1] < 2000;
}
"""


def compiled(tmp_path, source):
    (tmp_path / "strided.cpp").write_text(source)
    csrc = os.path.join(os.path.dirname(B.__file__), "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", csrc, str(tmp_path / "strided.cpp"), "-o", str(tmp_path / "strided")], check=True, timeout=120)
    r = subprocess.run([str(tmp_path / "strided")], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_rows_that_share_elements_among_themselves(tmp_path):
    compiled(tmp_path, STRIDED)


def test_outputs_that_share_elements_among_themselves_are_refused():
    far = 1 << 30
    for s in ([0, 1280, 128], [5120, 0, 128], [5120, 1280, 0], [5120, 1280, 120], [1280, 1280, 128], [5112, 1280, 128]):
        p = rparams(q_out_stride=s, k_out_stride=s, h_kv=4)
        assert apply(p, q_out=far, k=None, k_out=None) == -1 and apply(p, q=None, q_out=None, k_out=far) == -1, s
    far = dict(q=far, q_out=2 * far, k_new=3 * far, v_new=4 * far)
    for s in ([0, 128], [1024, 0], [1024, 120], [1016, 128], [256, 128]):      # 7 rows of 8 heads
        assert call4("rotary", params(o_stride=s), plan(), **far) == -1, s
        assert call4("append", params4(o_stride=s), plan(), **far) == -1, s
        assert call4("attend", params4(o_stride=s)) == -1, s
    n = dict(n=0)                                                # nothing else is wrong but the workspace
    assert call4("attend", params4(o_stride=[1024, 128]), **n) == call4("attend", params4(o_stride=[128, 896]), **n) == -3
    assert call4("attend", params4(n_rows=1, o_stride=[0, 128]), **n) == -3


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_tensors_that_share_elements_are_told_by_the_library(tmp_path):
    compiled(tmp_path, MEET)


def test_rotary_outputs_over_what_is_read_are_refused_by_the_library():
    """2 sequences of 4 and 2 heads of 128, 10 tokens, bf16; queries and keys as slices [tokens, heads, d] of one tensor of 8 heads, or of
    sequences inside of a token's row."""
    far, row = 1 << 30, 8 * 128
    fused = [10 * row, 128, row]
    st = dict(q_stride=fused, q_out_stride=fused, k_stride=fused, k_out_stride=fused)
    at = lambda heads: far + heads * 256  # noqa: E731
    for q, q_out, k, k_out in ((at(0), at(1), None, None), (at(0), at(0), at(3), at(3)), (at(0), 2 * far, at(4), 2 * far + 256), (at(0), at(4), at(6), 2 * far),
                               (at(0), 2 * far, at(6), at(3)), (at(0), at(4), at(3), 2 * far), (None, None, at(4), at(5))):
        assert apply(rparams(**st), q=q, q_out=q_out, k=k, k_out=k_out) == -1, (q, q_out, k, k_out)
    inner = [4 * 128, 128, 5 * 4 * 128]                          # [tokens, 5 sequences, 4 heads, d]: the second sequence of q is the first of k
    p = rparams(q_stride=inner, q_out_stride=inner, k_stride=inner, k_out_stride=inner)
    assert apply(p, q=far, q_out=far, k=far + 4 * 256, k_out=far + 4 * 256) == -1


def test_queries_turned_into_another_slice_of_their_tensor():
    """Apart from the queries, though in their span: accepted by appends into pages of either kind."""
    c, full, r = cache4(), B.PagedCache.allocate(2, 2, 8, 16, 64, 4, "cpu"), B.make_rotary(64, "cpu")
    p, fp, start = B.make_paged4_params(c, 3, 4), B.make_paged_params(full, 3, 4), torch.zeros(3, dtype=torch.int32)
    x = torch.zeros((3, 12, 64), dtype=torch.bfloat16)
    each = torch.zeros((3, 4, 4, 64), dtype=torch.bfloat16)      # (q, k, v, turned q) of each head side by side
    for q, q_out, meet in ((x[:, :4], x[:, 4:8], False), (x[:, 4:8], x[:, :4], False), (x[:, :4], x[:, 3:7], True), (x[:, 8:], x[:, 5:9], True),
                           (each[:, :, 0], each[:, :, 3], False), (each.view(3, 4, 256)[..., 32:96], each[:, :, 1], True)):
        for f in (lambda: B.dash_paged4_append(p, c, x[:, 8:10], x[:, 10:], start, rotary=r, q=q, q_out=q_out),
                  lambda: B.dash_paged_append_rotary(fp, full, r, x[:, 8:10], x[:, 10:], start, q=q, q_out=q_out)):
            with pytest.raises(B.DashError, match="overlap" if meet else "GPU"):
                f()
        with pytest.raises(B.DashError, match="overlap" if meet else "GPU"):
            B.dash_rotary(r, q.transpose(0, 1)[None], q_out.transpose(0, 1)[None])


def test_a_plans_scale_is_held_in_64_bits():
    for mscale in (1.2, 0.1, 1.0 + 2.0 ** -40):
        assert B.make_rotary(64, "cpu", mscale=mscale).plan.mscale == mscale
    for mscale in (1e39, 1e-50, -0.1):                           # no float
        assert apply(r=plan(mscale=mscale)) == -1


def test_turns_are_the_nearest_fractions():
    """A table off by more than half of its last bit would be off by more than |position| 2^-65 turns.  113 bits leave a theta of 2^30 2^-19 units of that bit."""
    D, most = decimal.Decimal, decimal.Decimal("0.50001")
    near = lambda want, got: abs((want * TURN - got).remainder_near(TURN)) <= most  # noqa: E731
    for rot in range(16, 144, 16):
        for base in (10000.0, 500000.0, 1e6, 10.0, 0.5, 1.0, 123456.789):
            rc, got = turns(rot, base=base)
            assert rc == 0 and all(near(t / R.TWO_PI, g) for t, g in zip(R.thetas(rot, base), got)), (rot, base)
        theta, f = R.thetas(rot), D(8)
        for scaling, want in ((1, [t / f for t in theta]), (2, [((D(10000).ln() + f.ln() * rot / (rot - 2)) * -2 * i / rot).exp() for i in range(rot // 2)]),
                              (3, [t * (c + (1 - c) / f) for t, c in ((t, min(max((D(8192) * t / R.TWO_PI - 1) / 31, D(0)), D(1))) for t in theta)])):
            rc, got = turns(rot, scaling=scaling, factor=8.0, original=8192.0, low=1.0, high=32.0)
            assert rc == 0 and all(near(t / R.TWO_PI, g) for t, g in zip(want, got)), (rot, scaling)
    gen = torch.Generator().manual_seed(1)
    freq = [1.0, 3.0, 100.0, -100.0, 0.1, 2.0 ** 30, -(2.0 ** 30 - 0.3), 1e-9, 5e-324, 0.0, 2 * math.pi] + (torch.randn(37, generator=gen, dtype=torch.float64) * 1000).tolist()
    rc, got = turns(96, freq=freq)
    assert rc == 0 and all(near(D(f) / R.TWO_PI % 1, g) for f, g in zip(freq, got))
    for huge in (1e300, -1e22):                                  # finite: a fraction, whichever
        assert turns(16, freq=[huge] * 8)[0] == 0
