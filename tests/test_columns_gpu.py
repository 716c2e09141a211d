"""Learned columns on the GPU against the fp64 oracle: dropout, lookup, the order of ids, the
table's gradient, the loss at given z; lengths, widths, strides, alignments, streams and
captured graphs.

Tolerances: of a lookup or a dropout 2 half steps of fp32 (scale times 1 / (1 - p), then the
product) and half a step of the result's type; of sums the oracle's bounds on fp32
arithmetic."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import ks_columns as o
from oracle import ks_fit as of
from paper_2606_28565_amd import abi

pytestmark = pytest.mark.gpu
NFAM = abi.NFAM
SEED = 0x1234_5678_9ABC_DEF1


def torch_type(t):
    import torch
    return torch.bfloat16 if t == "bf16" else torch.float32


def columns(n, cols, ld, shift, t, fill=-77.0):
    """A buffer and the columns of it from ``shift`` on that a call takes."""
    import torch
    buf = torch.full((n * ld + shift + 8,), fill, dtype=torch_type(t), device="cuda")
    return buf, buf[shift:shift + n * ld].view(n, ld)[:, :cols]


def rnd(n, cols, ld, shift, t, seed=3):
    import torch
    buf, x = columns(n, cols, ld, shift, t)
    x.copy_(torch.randn(n, cols, generator=torch.Generator().manual_seed(seed)))
    return x


def untouched(buf, view, fill=-77.0):
    """Whether nothing but the view's elements was written."""
    import torch
    seen = torch.zeros_like(buf, dtype=torch.bool)
    seen.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(True)
    return bool((buf[~seen] == fill).all())


def f64(t):
    return t.double().cpu().numpy()


def near(got, want, t):
    got, want = np.asarray(got), np.asarray(want)
    assert (np.abs(got - want) <= (2 * o.EPS + o.HALF[t]) * (1 + 2.0 ** -7) * np.abs(want)).all()


# ------------------------------------------------------------------ dropout
def run_dropout(x, y, p=0.25, site=1, step=5, step_dev=None, seed=SEED, stream=None):
    import torch
    abi.ks_dropout(abi.drop(p, seed, site, step, step_dev), abi.matrix(x), abi.matrix(y),
                   abi.current_stream() if stream is None else stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 16, 31, 67, 256, 2049, 4100])
def test_dropout_widths(t, cols):
    for n, pad, shift in ((1, 0, 0), (37, 0, 0), (300, 3, 1), (257, 8, 0)):
        x = rnd(n, cols, cols + pad, shift, t)
        buf, y = columns(n, cols, cols + pad, shift, t)
        run_dropout(x, y)
        want = o.drop(f64(x), 0.25, SEED, 1, 5)
        got = f64(y)
        assert ((got == 0) == (want == 0)).all()
        near(got, want, t)
        assert untouched(buf, y)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 1e-9, 0.1, 0.5, 0.999, 1.0])
def test_dropout_shares(p):
    """2^-17 rounds up to one step of the share; p = 1 leaves zeros."""
    x = rnd(400, 40, 40, 0, "f32")
    buf, y = columns(400, 40, 40, 0, "f32")
    run_dropout(x, y, p)
    near(f64(y), o.drop(f64(x), p, SEED, 1, 5), "f32")


def test_dropout_of_what_is_not_finite():
    """What is dropped is 0 whatever it was, what stays goes through."""
    import torch
    x = rnd(64, 24, 24, 0, "f32")
    x[::3] = float("nan")
    x[1::3] = float("inf")
    _, y = columns(64, 24, 24, 0, "f32")
    run_dropout(x, y, 0.5)
    k = torch.from_numpy(o.keep(np.arange(64), 24, 0.5, SEED, 1, 5)[0]).cuda()
    assert (y[~k] == 0).all() and y[k][:0].numel() == 0
    assert torch.isnan(y[::3][k[::3]]).all() and (y[1::3][k[1::3]] == float("inf")).all()


def test_each_word_of_the_counter_and_the_key_counts():
    x = rnd(200, 16, 16, 0, "f32")
    seen = []
    for seed, site, step in ((1, 0, 0), (1 << 32, 0, 0), (1, 1, 0), (1, 0, 1), ((1 << 64) - 1, (1 << 32) - 1, (1 << 32) - 1)):
        _, y = columns(200, 16, 16, 0, "f32")
        run_dropout(x, y, 0.5, site, step, seed=seed)
        near(f64(y), o.drop(f64(x), 0.5, seed, site, step), "f32")
        seen.append((f64(y) != 0).tobytes())
    assert len(set(seen)) == len(seen)


@pytest.mark.parametrize("t,ld", [("f32", 32), ("bf16", 35)])
def test_dropout_in_place_and_beside(t, ld):
    """x itself, and other columns of its buffer."""
    import torch
    x = rnd(500, 13, ld, 0, t)
    want = o.drop(f64(x), 0.25, SEED, 1, 5)
    buf = torch.full((500, ld), -77.0, dtype=x.dtype, device="cuda")
    buf[:, :13] = x
    run_dropout(buf[:, :13], buf[:, ld - 13:])
    near(f64(buf[:, ld - 13:]), want, t)
    assert (buf[:, :13] == x).all() and (buf[:, 13:ld - 13].float() == -77).all()
    run_dropout(buf[:, :13], buf[:, :13])
    near(f64(buf[:, :13]), want, t)
    assert (buf[:, 13:ld - 13].float() == -77).all()


def test_the_step_is_read_on_the_device():
    import torch
    x = rnd(300, 16, 16, 0, "f32")
    count = torch.tensor([41], dtype=torch.int32, device="cuda")
    _, y = columns(300, 16, 16, 0, "f32")
    run_dropout(x, y, step=7, step_dev=count)
    near(f64(y), o.drop(f64(x), 0.25, SEED, 1, 41), "f32")


def test_dropout_is_its_own_gradient():
    """The same struct on dy of another type and layout drops the same elements."""
    x, dy = rnd(130, 21, 21, 0, "f32"), rnd(130, 21, 32, 1, "bf16", 8)
    _, y = columns(130, 21, 21, 0, "f32")
    _, dx = columns(130, 21, 29, 0, "bf16")
    run_dropout(x, y)
    run_dropout(dy, dx)
    assert ((f64(y) == 0) == (f64(dx) == 0)).all()


# ------------------------------------------------------------------ lookup
def make_ids(n, v, seed=1, kind="skew"):
    """int32 ids: a few take most rows, some rows have none (-1) or one beyond the table."""
    import torch
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        ids = torch.full((n,), v // 2)
    elif kind == "none":
        ids = torch.full((n,), -1)
    elif kind == "all":
        ids = torch.randperm(n, generator=g) % v
    else:
        ids = (v * torch.rand(n, generator=g, dtype=torch.float64) ** 3).long().clamp(max=v - 1)
        bad = torch.rand(n, generator=g)
        ids = torch.where(bad < 0.02, -1, torch.where(bad < 0.04, v, ids))
    return ids.to(torch.int32).cuda()


def run_embed(table, scale, ids, y, drop=None, stream=None):
    import torch
    abi.ks_embed(abi.matrix(table), scale, ids.data_ptr(), None if drop is None else abi.drop(drop[0], drop[1], drop[2], drop[3]),
                 abi.matrix(y), abi.current_stream() if stream is None else stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("t_in", ["f32", "bf16"])
@pytest.mark.parametrize("t_out", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [1, 3, 8, 15, 16, 67, 1000, 4096])
@pytest.mark.parametrize("drop", [None, (0.3, SEED, 2, 9)])
def test_lookup(t_in, t_out, dim, drop):
    for n, v, pad, shift in ((1, 1, 0, 0), (130, 7, 16, 1), (1000, 300, 0, 0)):
        table = rnd(v, dim, dim + pad, shift, t_in, 4)
        ids = make_ids(n, v)
        buf, y = columns(n, dim, dim + pad, shift, t_out)
        run_embed(table, 1.7, ids, y, drop)
        near(f64(y), o.embed(f64(table), 1.7, ids.cpu().numpy(), drop), t_out)
        assert untouched(buf, y)


def test_ids_beyond_the_table():
    """2^32 - 1, n_ids and far ones give zeros; a table without rows gives only zeros."""
    import torch
    table = rnd(5, 24, 24, 0, "f32")
    table.fill_(3.0)
    ids = torch.tensor([0, -1, 4, 5, 6, 2 ** 31 - 1, -2 ** 31, 3], dtype=torch.int32, device="cuda")
    _, y = columns(8, 24, 24, 0, "f32")
    run_embed(table, 1.0, ids, y)
    assert y[:, 0].tolist() == [3, 0, 3, 0, 0, 0, 0, 3]
    run_embed(table[:0], 1.0, ids, y)
    assert (y == 0).all()


def test_values_that_are_not_finite_stay_in_their_rows():
    import torch
    table = rnd(6, 16, 16, 0, "f32")
    table[2] = float("nan")
    table[3] = float("inf")
    ids = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device="cuda")
    _, y = columns(4, 16, 16, 0, "f32")
    run_embed(table, -2.0, ids, y)
    assert torch.isnan(y[1]).all() and (y[2] == -float("inf")).all() and torch.isfinite(y[[0, 3]]).all()


# ------------------------------------------------------------------ order of ids
def run_order(ids, v, stream=None):
    import torch
    order = abi.id_order(ids.numel(), v)
    need = abi.ks_embed_sort_workspace_bytes(order)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    for t in order.t.values():
        t.fill_(-5)
    abi.ks_embed_sort(ids.data_ptr() if ids.numel() else None, order, ws.data_ptr(), need, abi.current_stream() if stream is None else stream)
    torch.cuda.synchronize()
    return order


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 1023, 1024, 1025, 4095, 4096, 4097, 8192, 8193, 16_384, 16_385, 20_011, 65_536, 65_537, 300_007, 1_100_003])
@pytest.mark.parametrize("v", [1, 2, 67, 255, 256, 1023, 1024, 5000, 131_072, (1 << 20) + 3])
def test_order(n, v):
    ids = make_ids(n, v, n + v)
    got = run_order(ids, v)
    row, key, off = o.order(ids.cpu().numpy(), v)
    for name, want in (("row", row), ("id", key), ("off", off)):
        assert (got.t[name].cpu().numpy() == want).all(), name


@pytest.mark.parametrize("kind", ["one", "none", "all"])
@pytest.mark.parametrize("n,v", [(5000, 9), (50_000, 3000), (9000, 1 << 22), (16_384, 20_000), (4097, 5000)])
def test_order_of_other_ids(kind, n, v):
    ids = make_ids(n, v, 1, kind)
    got = run_order(ids, v)
    row, key, off = o.order(ids.cpu().numpy(), v)
    for name, want in (("row", row), ("id", key), ("off", off)):
        assert (got.t[name].cpu().numpy() == want).all(), name


def test_order_of_many_rows():
    """More rows than 4096 chunks of keys, four digits."""
    import torch
    n, v = 17_000_003, (1 << 30) + 5
    g = torch.Generator("cuda").manual_seed(1)
    ids = torch.randint(0, 3000, (n,), generator=g, device="cuda", dtype=torch.int32)
    got = run_order(ids, 3000)
    want, row = torch.sort(ids, stable=True)
    assert (got.t["row"].long() == row).all() and (got.t["id"] == want).all()
    ids = torch.randint(0, v, (20_000,), generator=g, device="cuda", dtype=torch.int32)
    order = abi.id_order(20_000, v)
    ws = torch.empty(abi.ks_embed_sort_workspace_bytes(order), dtype=torch.uint8, device="cuda")
    abi.ks_embed_sort(ids.data_ptr(), order, ws.data_ptr(), ws.numel(), abi.current_stream())
    want, row = torch.sort(ids, stable=True)
    assert (order.t["row"].long() == row).all() and (order.t["id"] == want).all()
    at = torch.tensor([0, 1, v // 3, v // 2, v - 1, v], device="cuda")
    assert (order.t["off"][at].long() == torch.searchsorted(want, at.to(torch.int32))).all()


# ------------------------------------------------------------------ the table's gradient
def run_back(order, dy, grad, scale=1.0, drop=None, stream=None, ws=None):
    import torch
    m = abi.matrix(dy)
    need = abi.ks_embed_backward_workspace_bytes(order, m)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
    abi.ks_embed_backward(order, scale, m, None if drop is None else abi.drop(drop[0], drop[1], drop[2], drop[3]), abi.matrix(grad),
                          ws.data_ptr(), need, abi.current_stream() if stream is None else stream)
    torch.cuda.synchronize()


def check_back(n, v, dim, t="f32", pad=0, shift=0, scale=1.0, drop=None, kind="skew", positive=False):
    ids = make_ids(n, v, 2, kind)
    dy = rnd(n, dim, dim + pad, shift, t, 6)
    if positive:
        dy.abs_()
    buf, grad = columns(v, dim, dim + pad, shift, "f32")
    run_back(run_order(ids, v), dy, grad, scale, drop)
    want, bound = o.embed_back(ids.cpu().numpy(), v, f64(dy), scale, drop)
    off = np.abs(f64(grad) - want)
    assert (off <= bound).all(), (n, v, dim, float((off - bound).max()))
    assert untouched(buf, grad)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [1, 3, 8, 15, 16, 67, 200, 1000, 2048, 2056, 4100])
@pytest.mark.parametrize("drop", [None, (0.3, SEED, 2, 9)])
def test_gradient_widths(t, dim, drop):
    for n, v, pad, shift in ((1, 1, 0, 0), (700, 9, 5, 1), (1500, 900, 0, 0)):
        check_back(n, v, dim, t, pad, shift, 1.3, drop)


@pytest.mark.parametrize("n", [0, 1, 2, 127, 128, 129, 130, 513, 1536, 1537, 2047, 2048, 2049, 4099, 33_333, 300_007])
@pytest.mark.parametrize("v,dim", [(1, 16), (67, 16), (3000, 5), (5, 67)])
def test_gradient_lengths(n, v, dim):
    """Ids that begin and end inside, at and across the groups and parts of the order; one
    part and more."""
    check_back(n, v, dim)


@pytest.mark.parametrize("kind", ["one", "none", "all"])
@pytest.mark.parametrize("n,v,dim", [(700, 3, 40), (40_000, 60, 16), (3000, 4000, 24)])
def test_gradient_of_other_ids(kind, n, v, dim):
    check_back(n, v, dim, kind=kind, drop=(0.5, SEED, 0, 1))


def test_gradient_of_ids_as_long_as_a_part():
    """Every id exactly 128, 129, 2048 or 2047 rows."""
    import torch
    for each in (128, 129, 2047, 2048, 2049):
        ids = torch.arange(6, dtype=torch.int32).repeat(each)[torch.randperm(6 * each, generator=torch.Generator().manual_seed(2))].cuda()
        dy = rnd(6 * each, 16, 16, 0, "f32")
        _, grad = columns(6, 16, 16, 0, "f32")
        run_back(run_order(ids, 6), dy, grad)
        want, bound = o.embed_back(ids.cpu().numpy(), 6, f64(dy), 1.0)
        assert (np.abs(f64(grad) - want) <= bound).all(), each


def test_gradient_of_long_sums_of_one_sign():
    check_back(2_000_003, 67, 16, positive=True)
    check_back(2_000_003, 1, 7, "bf16", positive=True)


def test_gradient_gives_the_same_bits_again():
    import torch
    ids = make_ids(200_000, 100)
    dy = rnd(200_000, 19, 19, 0, "bf16")
    got = []
    for _ in range(3):
        _, grad = columns(100, 19, 19, 0, "f32")
        run_back(run_order(ids, 100), dy, grad, drop=(0.1, 5, 6, 7))
        got.append(grad.clone())
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_gradient_of_what_is_not_finite():
    """It reaches its id's row alone; a row without an id adds nothing, whatever it holds,
    nor does what was dropped."""
    import torch
    n = 1000
    ids = torch.arange(n, dtype=torch.int32).remainder(10).cuda()
    ids[7] = -1
    dy = rnd(n, 16, 16, 0, "f32")
    dy[7] = float("nan")
    dy[13, 2] = float("inf")
    _, grad = columns(10, 16, 16, 0, "f32")
    order = run_order(ids, 10)
    run_back(order, dy, grad)
    bad = ~torch.isfinite(grad)
    assert bad[3, 2] and int(bad.sum()) == 1
    k = o.keep([13], 16, 0.5, SEED, 0, 0)[0][0]
    dy[13] = float("nan")
    run_back(order, dy, grad, drop=(0.5, SEED, 0, 0))
    bad = ~torch.isfinite(grad)
    assert (bad[3].cpu().numpy() == k).all() and int(bad.sum()) == int(k.sum())


def test_an_order_of_something_else_stays_inside():
    """Offsets and rows that no call made: the sums are of something else, and nothing but
    the gradient's rows is written (every access is checked against the sizes)."""
    import torch
    n, v = 5000, 40
    order = run_order(make_ids(n, v), v)
    dy = rnd(n, 16, 16, 0, "f32")
    g = torch.Generator("cuda").manual_seed(3)
    for name in ("row", "off", "id"):
        t = order.t[name]
        t.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, t.shape, generator=g, device="cuda"))
        buf, grad = columns(v, 16, 20, 3, "f32")
        run_back(order, dy, grad)
        assert untouched(buf, grad)


# ------------------------------------------------------------------ the loss at given z
def run_eta(z, eta, weight, off, huber, stream=None, dz=None):
    import torch
    loss = torch.full((NFAM,), float("nan"), device="cuda")
    dz = torch.full_like(z, float("nan")) if dz is None else dz
    f = abi.family_offsets(off)
    need = abi.ks_eta_loss_workspace_bytes(f)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    abi.ks_eta_loss(f, z.data_ptr() if z.numel() else None, abi.eta_target(eta, weight, huber), loss.data_ptr(),
                    dz.data_ptr() if z.numel() else None, ws.data_ptr(), need, abi.current_stream() if stream is None else stream)
    torch.cuda.synchronize()
    return loss, dz


def family_split(n, kind="mixed"):
    if kind == "one":
        return [0] * 5 + [n] * 6
    if kind == "last":
        return [0] * 10 + [n]
    cut = np.floor(np.cumsum([5, 0, 1, 2, 2, 4, 1, 0, 1, 1]) / 17 * n).astype(int)
    return [0] + [int(v) for v in cut[:-1]] + [n]


def make_eta(n, seed=4, shift=0):
    import torch
    g = torch.Generator().manual_seed(seed)

    def off_grid(v):
        room = torch.zeros(n + shift, device="cuda")
        room[shift:] = v
        return room[shift:]
    eta = 1 + torch.exp(0.7 * torch.randn(n, generator=g) - 1)
    kind = torch.rand(n, generator=g)
    for lo, bad in ((0.0, float("nan")), (0.02, 0.0), (0.04, -1.0), (0.06, float("inf"))):
        eta = torch.where((kind >= lo) & (kind < lo + 0.02), bad, eta)
    weight = 0.5 + torch.rand(n, generator=g)
    for lo, bad in ((0.9, 0.0), (0.92, -1.0), (0.94, float("nan")), (0.96, float("inf"))):
        weight = torch.where((kind >= lo) & (kind < lo + 0.02), bad, weight)
    return off_grid(1.5 * torch.randn(n, generator=g)), off_grid(eta), off_grid(weight)


def check_eta(z, eta, weight, off, huber, got):
    loss, dz = f64(got[0]), f64(got[1])
    z, eta = f64(z), f64(eta)
    weight = None if weight is None else f64(weight)
    for f in range(NFAM):
        r = slice(off[f], off[f + 1])
        w = None if weight is None else weight[r]
        want, want_dz = of.eta_loss(z[r], eta[r], w, huber)
        b, b_dz = o.eta_bounds(z[r], eta[r], w, huber, want, want_dz)
        assert abs(loss[f] - want) <= b, f
        assert (np.abs(dz[r] - want_dz) <= b_dz).all(), f
        assert (dz[r][of.counted(eta[r], w) == 0] == 0).all(), f


@pytest.mark.parametrize("n", [0, 1, 2, 3, 17, 100, 1023, 1025, 4099, 20_000, 70_001, 300_007])
@pytest.mark.parametrize("kind", ["mixed", "one", "last"])
@pytest.mark.parametrize("huber,weighted", [(float("inf"), False), (0.3, True)])
def test_eta_loss(n, kind, huber, weighted):
    z, eta, weight = make_eta(n)
    off = family_split(n, kind)
    weight = weight if weighted else None
    check_eta(z, eta, weight, off, huber, run_eta(z, eta, weight, off, huber))


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_eta_loss_off_the_16_byte_grid(shift):
    z, eta, weight = make_eta(5003, shift=shift)
    off = family_split(5003)
    check_eta(z, eta, weight, off, 0.2, run_eta(z, eta, weight, off, 0.2))


def test_eta_loss_over_z():
    """dz in z's place; rows that do not count get 0 whatever their z."""
    import torch
    for n in (3000, 200_001):
        z, eta, weight = make_eta(n)
        off = family_split(n)
        want = run_eta(z, eta, weight, off, 0.5)
        z[torch.isnan(eta)] = float("nan")
        got = run_eta(z, eta, weight, off, 0.5, dz=z)
        assert torch.equal(got[0], want[0]) and torch.equal(z, want[1])


def test_eta_loss_of_far_z():
    """Overflow on neither side; a family without rows that count loses 0."""
    import torch
    z = torch.tensor([-1e4, -200.0, -90.0, 0.0, 90.0, 200.0, 1e4] * 10, device="cuda")
    off = [7 * i for i in range(NFAM + 1)]
    eta = torch.full((70,), 2.0, device="cuda")
    eta[14:21] = float("nan")
    loss, dz = run_eta(z, eta, None, off, 1.0)
    assert torch.isfinite(loss).all() and torch.isfinite(dz).all() and loss[2] == 0
    check_eta(z, eta, None, off, 1.0, (loss, dz))


def test_eta_loss_is_ks_gated_loss():
    """ks_gated_forward's z through the loss and ks_gated_backward: ks_gated_loss's values."""
    import torch
    n, inp, hid = 5000, 32, 64
    g = torch.Generator().manual_seed(2)
    w = {k: (0.3 * torch.randn(*s, generator=g)).cuda() for k, s in
         (("w1", (NFAM, hid, inp)), ("w2", (NFAM, hid, inp)), ("w3", (NFAM, hid)), ("b3", (NFAM,)))}
    x = torch.rand(n, inp, generator=g).cuda()
    off = family_split(n)
    _, eta, weight = make_eta(n)
    hd, rows, tgt = abi.gated_heads(**w), abi.feature_rows(x, off), abi.eta_target(eta, weight, 0.5)
    ws = torch.empty(abi.ks_gated_workspace_bytes(hd, rows), dtype=torch.uint8, device="cuda")
    one = {k: torch.empty_like(v) for k, v in w.items()}
    two = {k: torch.empty_like(v) for k, v in w.items()}
    loss, z = torch.empty(NFAM, device="cuda"), torch.empty(n, device="cuda")
    s = abi.current_stream()
    abi.ks_gated_loss(hd, rows, tgt, loss.data_ptr(), None, abi.gated_grad(**one), ws.data_ptr(), ws.numel(), s)
    abi.ks_gated_forward(hd, rows, z.data_ptr(), s)
    got, dz = run_eta(z, eta, weight, off, 0.5)
    abi.ks_gated_backward(hd, rows, dz.data_ptr(), abi.gated_grad(**two), ws.data_ptr(), ws.numel(), s)
    torch.cuda.synchronize()
    # the same terms in another order of sums: 16 roundings of a sum's magnitude
    assert torch.allclose(got, loss, rtol=16 * o.EPS, atol=0)
    for k in one:
        size = float(one[k].abs().max())
        assert float((one[k] - two[k]).abs().max()) <= 64 * o.EPS * size, k


# ------------------------------------------------------------------ streams, graphs, far ends
def test_other_stream_and_two_at_once():
    """Two streams, a workspace each; ids, tables and gradients of their own."""
    import torch
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = []
    for i, s in enumerate(streams):
        n, v, dim = 50_000 + i, 90 + 900 * i, 16 + 8 * i
        ids, dy = make_ids(n, v, i), rnd(n, dim, dim, 0, "f32", i)
        order, grad = abi.id_order(n, v), torch.full((v, dim), float("nan"), device="cuda")
        sort_ws = torch.empty(abi.ks_embed_sort_workspace_bytes(order), dtype=torch.uint8, device="cuda")
        ws = torch.empty(abi.ks_embed_backward_workspace_bytes(order, abi.matrix(dy)), dtype=torch.uint8, device="cuda")
        work.append((ids, order, dy, grad, sort_ws, ws))
    torch.cuda.synchronize()
    for _ in range(3):
        for (ids, order, dy, grad, sort_ws, ws), s in zip(work, streams):
            abi.ks_embed_sort(ids.data_ptr(), order, sort_ws.data_ptr(), sort_ws.numel(), s.cuda_stream)
            abi.ks_embed_backward(order, 1.0, abi.matrix(dy), None, abi.matrix(grad), ws.data_ptr(), ws.numel(), s.cuda_stream)
    torch.cuda.synchronize()
    for ids, order, dy, grad, _, _ in work:
        want, bound = o.embed_back(ids.cpu().numpy(), order.n_ids, f64(dy), 1.0)
        assert (np.abs(f64(grad) - want) <= bound).all()


def test_captured_calls_replay():
    """A pass of all calls captured, replayed with other ids, values and steps, against the
    eager calls between the replays."""
    import torch
    n, v, dim = 9000, 70, 16
    ids, table = make_ids(n, v), rnd(v, dim, dim, 0, "f32")
    rows = torch.zeros(n, 32, device="cuda")
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    drop = abi.drop(0.2, SEED, 3, step_dev=count)
    order = abi.id_order(n, v)
    grad = torch.zeros(v, dim, device="cuda")
    z, eta, weight = make_eta(n)
    off, tgt = abi.family_offsets(family_split(n)), abi.eta_target(eta, weight, 0.5)
    loss, dz = torch.zeros(NFAM, device="cuda"), torch.zeros(n, device="cuda")
    y, x = abi.matrix(rows[:, 16:]), abi.matrix(rows[:, :15])
    need = (abi.ks_embed_sort_workspace_bytes(order), abi.ks_embed_backward_workspace_bytes(order, y), abi.ks_eta_loss_workspace_bytes(off))
    ws = [torch.empty(b, dtype=torch.uint8, device="cuda") for b in need]

    def call():
        s = abi.current_stream()
        abi.ks_embed(abi.matrix(table), 1.5, ids.data_ptr(), drop, y, s)
        abi.ks_dropout(drop, y, abi.matrix(rows[:, :16]), s)
        abi.ks_embed_sort(ids.data_ptr(), order, ws[0].data_ptr(), need[0], s)
        abi.ks_embed_backward(order, 1.0, y, drop, abi.matrix(grad), ws[1].data_ptr(), need[1], s)
        abi.ks_eta_loss(off, z.data_ptr(), tgt, loss.data_ptr(), dz.data_ptr(), ws[2].data_ptr(), need[2], s)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        ids.copy_(make_ids(n, v, 10 + i))
        table.mul_(0.9)
        z.mul_(0.8)
        count.add_(1)
        g.replay()
        torch.cuda.synchronize()
        seen = [t.clone() for t in (rows, grad, loss, dz, *order.t.values())]
        call()   # eager, between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(seen, (rows, grad, loss, dz, *order.t.values()))), i
    near(f64(rows[:, 16:]), o.embed(f64(table), 1.5, ids.cpu().numpy(), (0.2, SEED, 3, 4)), "f32")


def test_offsets_past_32_bits():
    """Rows 2^16 elements apart, over 10 GB: lookup, dropout and gradient as of near rows."""
    import torch
    n, ld, dim, v = 40_000, 1 << 16, 24, 3000
    far = torch.empty(n * ld, dtype=torch.float32, device="cuda").view(n, ld)[:, :dim]
    ids = make_ids(n, v)
    table = rnd(v, dim, dim, 0, "f32")
    near_y = torch.empty(n, dim, device="cuda")
    drop = (0.25, SEED, 1, 5)
    run_embed(table, 1.0, ids, near_y, drop)
    run_embed(table, 1.0, ids, far, drop)
    assert torch.equal(far, near_y)
    run_dropout(far, far)
    run_dropout(near_y, near_y)
    assert torch.equal(far, near_y)
    order = run_order(ids, v)
    grads = [torch.empty(v, dim, device="cuda") for _ in range(2)]
    run_back(order, far, grads[0], 1.0, drop)
    run_back(order, near_y, grads[1], 1.0, drop)
    assert torch.equal(*grads)


def test_more_blocks_than_a_launch_takes():
    """2^31 columns' blocks and more: 2.15e9 lanes in two launches, draws past 32 bits of
    elements."""
    import torch
    n = (1 << 31) - 1
    x = torch.ones(n, 1, dtype=torch.bfloat16, device="cuda")
    run_dropout(x, x, 0.5)
    for lo in (0, (1 << 31) - 70_000):
        rows = np.arange(lo, lo + 60_000)
        want = o.keep(rows, 1, 0.5, SEED, 1, 5)[0]
        assert ((f64(x[lo:lo + 60_000]) != 0) == want).all()
    share = sum(int((c != 0).sum()) for c in x.view(-1).split(1 << 28)) / n
    assert abs(share - 0.5) < 5 * 0.5 / np.sqrt(n)


def test_gradient_of_a_far_table():
    """A gradient of more than 2^32 elements: rows of the last ids, and zeros between."""
    import torch
    v, dim = 70_000, 1 << 16
    ids = torch.tensor([v - 1, 65_536, 65_537, v - 1, 0], dtype=torch.int32, device="cuda")
    dy = torch.arange(1, 6, device="cuda", dtype=torch.float32)[:, None].expand(5, dim).contiguous()
    grad = torch.full((v, dim), float("nan"), device="cuda")
    run_back(run_order(ids, v), dy, grad)
    want = torch.zeros(v, device="cuda")
    want[[0, 65_536, 65_537, v - 1]] = torch.tensor([5.0, 2.0, 3.0, 5.0], device="cuda")
    for lo in range(0, v, 10_000):
        assert (grad[lo:lo + 10_000] == want[lo:lo + 10_000, None]).all()


@pytest.mark.parametrize("dim,ld,shift", [(128, 128, 0), (127, 128, 0), (126, 132, 4), (129, 129, 0), (128, 128, 1)])
def test_gradient_of_a_large_table(dim, ld, shift):
    """Over 128 MiB, on the 16-byte grid and off it: all ids' rows and nothing else."""
    import torch
    v, n = 300_000, 2000
    g = torch.Generator().manual_seed(6)
    ids = torch.randint(0, v, (n,), generator=g).to(torch.int32)
    ids[:3] = torch.tensor([0, v - 1, v])
    ids = ids.cuda()
    dy = rnd(n, dim, dim, 0, "f32")
    order = run_order(ids, v)
    buf, grad = columns(v, dim, ld, shift, "f32")
    run_back(order, dy, grad)
    seen = torch.unique(ids[ids < v].long())
    want, bound = o.embed_back(ids.cpu().numpy(), v, f64(dy), 1.0)
    at = seen.cpu().numpy()
    assert (np.abs(f64(grad[seen]) - want[at]) <= bound[at]).all()
    rest = torch.ones(v, dtype=torch.bool, device="cuda")
    rest[seen] = False
    assert (grad[rest] == 0).all()
    assert untouched(buf, grad)


def test_tables_of_more_than_32_bits():
    """A table of more than 2^32 elements."""
    import torch
    v, dim = 70_000, 1 << 16
    table = torch.zeros(v, dim, dtype=torch.bfloat16, device="cuda")
    table[:, :3] = torch.arange(v, device="cuda").remainder(251)[:, None].to(torch.bfloat16)
    ids = torch.tensor([0, 1, 65_535, 65_536, 65_537, v - 1, v], dtype=torch.int32, device="cuda")
    y = torch.empty(7, dim, device="cuda")
    run_embed(table, 1.0, ids, y)
    want = [float(i % 251) for i in (0, 1, 65_535, 65_536, 65_537, v - 1)] + [0.0]
    assert y[:, 2].tolist() == want and (y[:, 3:] == 0).all()
