"""CPU-side tests of the paged cache's entry points: sizes, refusals before any launch, the binding's checks, and the plain
forms of the GPU tests against torch."""
import ctypes
import dataclasses
import math

import pytest
import torch

import paged_ref as R
from test_library_host import kernel_scratch
from paper_2605_18753_amd import binding as B


def params(**kw):
    p = B.dash_paged_params()
    base = dict(batch=4, h_q=8, h_kv=2, head_dim=128, dtype=B.DASH_BF16, causal=1, page_size=64, n_pages=100, max_pages=20, n_rows=7)
    base.update({k: v for k, v in kw.items() if not k.endswith("stride")})
    for k, v in base.items():
        setattr(p, k, v)
    d = p.head_dim
    p.q_stride[:] = p.o_stride[:] = [p.h_q * d, d]
    p.k_new_stride[:] = p.v_new_stride[:] = [p.h_kv * d, d]
    p.k_stride[:] = p.v_stride[:] = [p.h_kv * p.page_size * d, p.page_size * d, d]
    for k, v in kw.items():
        if k.endswith("stride"):
            getattr(p, k)[:] = v
    return p


def call(name, p, ws=4096, n=1 << 40, **kw):
    """The entry point with pointers that no launch may reach (the refusals come first)."""
    a = dict(k_new=256, v_new=256, q=256, k=256, v=256, o=256, lse=256, row_start=256, lens=256, table=256, weights=256, pos=256, seen=256,
             src=None, budget=100, sinks=4, recent=10, last=0)
    a.update(kw)
    lib, g = B.load_library(), a.get
    p = ctypes.byref(p)
    if name == "append":
        return lib.dash_paged_append(p, g("k_new"), g("v_new"), g("k"), g("v"), g("row_start"), g("lens"), g("table"), g("weights"), g("pos"), g("seen"), None)
    if name == "attend":
        return lib.dash_paged_attend(p, g("q"), g("k"), g("v"), g("row_start"), g("lens"), g("table"), g("o"), g("lse"), ws, n, None)
    if name == "weigh":
        return lib.dash_paged_weigh(p, g("q"), g("k"), g("row_start"), g("lens"), g("table"), g("lse"), g("last"), g("weights"), ws, n, None)
    return lib.dash_paged_evict(p, g("k"), g("v"), g("lens"), g("seen"), g("table"), g("weights"), g("pos"), g("budget"), g("sinks"), g("recent"),
                                g("src"), ws, n, None)


ALL = ("append", "attend", "weigh", "evict")


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -1), (dict(h_q=7), -1), (dict(h_kv=0), -1), (dict(dtype=2), -1), (dict(causal=2), -1), (dict(n_pages=0), -1),
    (dict(max_pages=0), -1), (dict(page_size=0), -1), (dict(reserved=1), -1), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1),
    (dict(k_stride=[16384, 8192, 120]), -1), (dict(v_stride=[16384, 8192, 124]), -1), (dict(k_stride=[-8, 8192, 128]), -1),
    (dict(head_dim=96), -2), (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=2048), -2),
    (dict(h_q=64, h_kv=2), -2), (dict(h_q=6, h_kv=2), -2), (dict(max_pages=1 << 20), -2), (dict(k_stride=[16384, 8192, 1 << 26]), -2),
    (dict(v_stride=[16384, 8192, 1 << 62]), -2), (dict(batch=1 << 20), -2),
])
def test_parameters_that_every_call_refuses(kw, code):
    for name in ALL:
        assert call(name, params(**kw)) == code, name
    n = ctypes.c_size_t(0)
    for f in (B.load_library().dash_paged_workspace_bytes, B.load_library().dash_paged_evict_workspace_bytes):
        assert f(ctypes.byref(params(**kw)), ctypes.byref(n)) == code
        assert f(ctypes.byref(params()), None) == -1 and f(None, ctypes.byref(n)) == -1


def test_parameters_of_the_packed_rows():
    for name in ("append", "attend", "weigh"):
        assert call(name, params(n_rows=0)) == -1 and call(name, params(n_rows=(1 << 28) + 1)) == -2
    for s in ("q_stride", "o_stride"):
        for bad in ([1024, 4], [-8, 128]):
            assert call("attend", params(**{s: bad})) == -1
    assert call("append", params(k_new_stride=[4, 128])) == -1 and call("append", params(v_new_stride=[256, -8])) == -1


@pytest.mark.parametrize("name,needed", [
    ("append", ("k_new", "v_new", "k", "v", "row_start", "lens", "table")), ("attend", ("q", "k", "v", "row_start", "lens", "table", "o")),
    ("weigh", ("q", "k", "row_start", "lens", "table", "lse", "weights")), ("evict", ("k", "v", "lens", "seen", "table", "weights", "pos")),
])
def test_null_and_misaligned_pointers(name, needed):
    for x in needed:
        assert call(name, params(), **{x: None}) == -1, x
    for x in set(needed) & {"k_new", "v_new", "q", "k", "v", "o"}:
        assert call(name, params(), **{x: 264}) == -1, x


def test_workspaces():
    n, e = B.paged_workspace_bytes(params()), B.paged_workspace_bytes(params(), evict=True)
    for name, need in (("attend", n), ("weigh", B.paged_workspace_bytes(params())), ("evict", e)):
        assert call(name, params(), ws=None) == -3 and call(name, params(), ws=4097) == -3
    assert call("attend", params(), n=0) == -3 and call("evict", params(), n=e - 1) == -3 and call("weigh", params(), n=0) == -3
    # the eviction's lists: a number a slot; of long caches also the keys, those picked out with their slots, and counts of every 4096
    assert 4 * 2 * 20 * 64 * 4 <= e <= 4 * 2 * 20 * 64 * 4 + 4096
    big = B.paged_workspace_bytes(params(max_pages=513), evict=True)
    assert 4 * 2 * 513 * 64 * 16 + 4 * 2 * 10 * 2048 * 4 <= big <= 4 * 2 * 513 * 64 * 16 + 4 * 2 * 10 * 2049 * 4 + 4096
    # one workspace serves every number of rows
    assert all(B.paged_workspace_bytes(params(n_rows=r)) == n for r in (1, 64, 5000, 1 << 20))


def test_eviction_budgets():
    for kw in (dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(budget=13), dict(sinks=1 << 30, recent=1 << 30, budget=1 << 30)):
        assert call("evict", params(), **kw) == -1, kw
    assert call("weigh", params(), last=-1) == -1


def test_the_binding_refuses_tensors_that_do_not_fit():
    c = B.PagedCache.allocate(2, 2, 8, 16, 64, 4, "cpu", evicting=True)
    p = B.make_paged_params(c, 3, 4)
    assert (p.batch, p.h_kv, p.h_q, p.page_size, p.n_pages, p.max_pages, p.head_dim, p.n_rows, p.dtype) == (2, 2, 4, 16, 8, 4, 64, 3, B.DASH_BF16)
    assert (c.table == -1).all() and (c.lens == 0).all()
    ws, start = torch.empty(1 << 20, dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)
    q, lse = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 4))
    good = dict(q=q, o=q.clone(), row_start=start, lse=lse)
    for bad in (dict(q=q[:2]), dict(q=q.float()), dict(o=q[:, :3]), dict(row_start=start.long()), dict(row_start=start[:2]),
                dict(lse=lse.double()), dict(lse=lse.t()), dict(q=torch.zeros((3, 4, 128), dtype=torch.bfloat16)[..., ::2])):
        a = {**good, **bad}
        with pytest.raises(B.DashError):
            B.dash_paged_attend(p, c, a["q"], a["row_start"], a["o"], ws, lse=a["lse"])
    with pytest.raises(B.DashError):
        B.dash_paged_evict(p, c, 8, ws, src=torch.zeros((2, 2, 9), dtype=torch.int32))
    with pytest.raises(B.DashError):
        B.dash_paged_weigh(p, c, q, start, None, ws)
    bare = B.PagedCache(c.k, c.v, c.table, c.lens)
    for f in (lambda: B.dash_paged_weigh(p, bare, q, start, lse, ws), lambda: B.dash_paged_evict(p, bare, 8, ws)):
        with pytest.raises(B.DashError):
            f()
    for k, v, t, n in ((c.k.half(), c.v.half(), c.table, c.lens), (c.k, c.v.float(), c.table, c.lens), (c.k, c.v, c.table.long(), c.lens),
                       (c.k, c.v, c.table, c.lens[:1]), (c.k[..., ::2], c.v[..., ::2], c.table, c.lens), (c.k, c.v[:4], c.table, c.lens)):
        with pytest.raises(B.DashError):
            B.make_paged_params(B.PagedCache(k, v, t, n), 3, 4)
    with pytest.raises(B.DashError, match="GPU"):               # nothing wrong but where the tensors lie
        B.dash_paged_attend(p, c, q, start, q.clone(), ws, lse=lse)
    assert list(p.q_stride) == [0, 0]                           # a call leaves the caller's parameters alone


def test_the_binding_refuses_the_parameters_of_another_cache():
    c = B.PagedCache.allocate(2, 2, 8, 16, 64, 4, "cpu", evicting=True)
    p = B.make_paged_params(c, 3, 4)
    q, start = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    fewer = {"k": c.k[:4], "v": c.v[:4], "table": c.table[:, :2].contiguous(), "lens": c.lens.long()}
    token = torch.zeros((8, 16, 2, 64), dtype=torch.bfloat16).transpose(1, 2)
    for field, x in (*fewer.items(), ("table", c.table[:1]), ("k", token), ("v", token), ("k", c.k.float())):
        other = dataclasses.replace(c, **{field: x})
        for f in (lambda: B.dash_paged_attend(p, other, q, start, q.clone(), ws), lambda: B.dash_paged_evict(p, other, 8, ws),
                  lambda: B.dash_paged_append(p, other, q[:, :2], q[:, 2:], start)):
            with pytest.raises(B.DashError, match="other sizes|fit each other|int32|pages"):
                f()
    with pytest.raises(B.DashError, match="GPU"):               # other tensors, alike
        B.dash_paged_attend(p, B.PagedCache(c.k.clone(), c.v.clone(), c.table.clone(), c.lens.clone()), q, start, q.clone(), ws)


def test_the_plain_forms_agree_with_torch():
    gen = torch.Generator().manual_seed(1)
    k, v = (torch.randn((6, 2, 16, 64), generator=gen, dtype=torch.float32) for _ in range(2))
    table = torch.tensor([[4, 1, 3], [0, 5, -1]], dtype=torch.int32)
    c = R.Cache(k, v, table, torch.tensor([40, 20], dtype=torch.int32), weights=torch.zeros((6, 2, 16)))
    q = torch.randn((9, 4, 64), generator=gen)
    start = torch.tensor([0, 5, 9], dtype=torch.int32)
    o, lse, tol, _ = R.attend(c, q, start, 2)
    w, _ = R.weigh(c, q, start, lse, 2)
    total = 0.0
    for b, (n, r0, r1) in enumerate(((40, 0, 5), (20, 5, 9))):
        flat = lambda x: x[table[b, :-(-n // 16)].long()].transpose(0, 1).reshape(2, -1, 64)[:, :n].double().repeat_interleave(2, 0)  # noqa: E731
        m = r1 - r0
        mask = torch.ones((m, n), dtype=torch.bool).tril(n - m)
        ref = torch.nn.functional.scaled_dot_product_attention(q[r0:r1].double().transpose(0, 1), flat(k), flat(v), attn_mask=mask)
        assert (ref.transpose(0, 1) - o[r0:r1]).abs().max() < 1e-12
        total += 4 * m
    assert abs(float(w.sum()) - total) < 1e-9 and (tol > 0).all()


def test_the_kernels_use_no_scratch_memory():
    scratch = {n: b for n, b in kernel_scratch(B.LIB_PATH).items() if "dash" in n and "paged_" in n}
    assert len(scratch) >= 20 and not {n: b for n, b in scratch.items() if b}


def test_the_binding_looks_at_a_tensor_that_is_assigned():
    c = B.PagedCache.allocate(2, 2, 8, 16, 64, 4, "cpu", evicting=True)
    p = B.make_paged_params(c, 3, 4)
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    for field, bad in (("weights", c.weights.double()), ("weights", c.weights[:4]), ("pos", c.pos.long()), ("pos", c.pos.transpose(1, 2)),
                       ("seen", c.seen[:1]), ("lens", c.lens.long()), ("v", c.v.float()), ("table", c.table.t())):
        good = getattr(c, field)
        setattr(c, field, bad)
        with pytest.raises(B.DashError, match="contiguous|pages"):
            B.dash_paged_evict(p, c, 8, ws)
        setattr(c, field, good)
    c.weights = c.weights.clone()
    with pytest.raises(B.DashError, match="GPU"):
        B.dash_paged_evict(p, c, 8, ws)


def test_the_binding_looks_at_the_tensors_of_every_call():
    """A tensor changed in place behind the first call (the same object, other sizes) is refused before anything reads by the old ones."""
    def fresh():
        c = B.PagedCache.allocate(2, 2, 8, 16, 64, 4, "cpu", evicting=True)
        p = B.make_paged_params(c, 3, 4)
        call = lambda: B.dash_paged_evict(p, c, 8, torch.empty(1 << 20, dtype=torch.uint8))  # noqa: E731
        with pytest.raises(B.DashError, match="GPU"):            # nothing wrong but where the tensors lie
            call()
        return c, p, call
    changes = {
        "k pages fewer": lambda c: setattr(c.k, "data", c.k[:4]), "v pages fewer": lambda c: c.v.resize_(4, 2, 16, 64),
        "k of another type": lambda c: setattr(c.k, "data", c.k.float()), "v strides": lambda c: setattr(c.v, "data", c.v.transpose(1, 2).contiguous().transpose(1, 2)),
        "lens": lambda c: c.lens.resize_(1), "table": lambda c: c.table.resize_(2, 2), "table of another order": lambda c: c.table.t_(),
        "weights": lambda c: c.weights.resize_(4, 2, 16), "weights of another type": lambda c: setattr(c.weights, "data", c.weights.double()),
        "pos": lambda c: setattr(c.pos, "data", c.pos.transpose(1, 2)), "seen": lambda c: setattr(c.seen, "data", c.seen.long()),
    }
    for name, change in changes.items():
        c, _, call = fresh()
        change(c)
        with pytest.raises(B.DashError, match="contiguous|pages|other sizes"):
            call()
    # and parameters whose sizes or strides are no longer the cache's
    for field, value in (("batch", 3), ("n_pages", 9), ("max_pages", 5), ("page_size", 32), ("h_kv", 4), ("head_dim", 128), ("dtype", B.DASH_F32)):
        _, p, call = fresh()
        setattr(p, field, value)
        with pytest.raises(B.DashError, match="other sizes"):
            call()
    for field in ("k_stride", "v_stride"):
        _, p, call = fresh()
        getattr(p, field)[2] = 128
        with pytest.raises(B.DashError, match="other sizes"):
            call()


@pytest.mark.parametrize("far", [(1 << 32) + 8, 1 << 31, -(1 << 32) + 8])
def test_the_binding_refuses_numbers_that_do_not_fit_32_bits(far):
    """They would be cut to their low 32 bits on the way: a budget of 2^32 + 8 tokens to one of 8."""
    c = B.PagedCache.allocate(2, 2, 8, 16, 64, 4, "cpu", evicting=True)
    p = B.make_paged_params(c, 8, 4)
    ws, start = torch.empty(1 << 20, dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)
    q, lse = torch.zeros((8, 4, 64), dtype=torch.bfloat16), torch.zeros((8, 4))
    for f in (lambda: B.dash_paged_evict(p, c, far, ws), lambda: B.dash_paged_evict(p, c, 8, ws, sinks=far), lambda: B.dash_paged_evict(p, c, 8, ws, recent=far),
              lambda: B.dash_paged_weigh(p, c, q, start, lse, ws, last=far), lambda: B.make_paged_params(c, far, 4), lambda: B.make_paged_params(c, 8, far)):
        with pytest.raises(B.DashError, match="32 bits"):
            f()


def test_the_binding_refuses_a_workspace_whose_elements_do_not_lie_in_a_row():
    """Its number of elements is not the bytes behind its address."""
    one = torch.empty(1, dtype=torch.uint8)
    for ws in (one.expand(1 << 30), torch.empty(1 << 12, dtype=torch.uint8)[::2]):
        with pytest.raises(B.DashError, match="contiguous"):
            B._ws_ptr(ws)
    assert B._ws_ptr(torch.empty(1 << 12, dtype=torch.uint8))[1] > (1 << 12) - 256


def test_fp32_attention_refuses_more_rows_than_a_launch_has_threads_for():
    """512 threads for 16 rows of a kv-head's group; threads behind 2^32 would be left out without an error."""
    def rc(n_rows, batch, h_q, h_kv, dtype=B.DASH_F32, name="attend"):
        p = params(n_rows=n_rows, batch=batch, h_q=h_q, h_kv=h_kv, head_dim=64, dtype=dtype)
        return call(name, p, ws=4096, n=0 if name == "attend" else 1 << 40, k=264 if name == "weigh" else 256)
    for case in (((1 << 24), 1, 16, 16), ((1 << 28), 1, 1, 1), ((1 << 23) - 1 << 4, 1, 1, 1), ((1 << 22), 1, 64, 4), ((1 << 23) - (1 << 20) << 4, 1 << 20, 1, 1)):
        assert rc(*case) == -2, case
    # the next smaller ones, and others of as many rows, come to the next check (the workspace's, the pages' alignment)
    for case in (((1 << 23) - 1 << 4) - 1, 1, 1, 1), (1 << 22, 1 << 20, 1, 1):
        assert rc(*case) == -3, case
    assert rc(1 << 24, 1, 16, 16, dtype=B.DASH_BF16) == -3 and rc(1 << 24, 1, 16, 16, name="weigh") == -1


def test_outputs_that_share_elements_among_themselves_are_refused():
    for s in ([0, 128], [1024, 0], [1024, 120], [1016, 128], [256, 128]):      # 7 rows of 8 heads
        assert call("attend", params(o_stride=s)) == -1, s
    assert call("attend", params(o_stride=[1024, 128]), n=0) == call("attend", params(o_stride=[128, 896]), n=0) == -3
    assert call("attend", params(n_rows=1, o_stride=[0, 128]), n=0) == -3
