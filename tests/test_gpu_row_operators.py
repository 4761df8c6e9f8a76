"""The operators on rows against plain forms in 64 bits: lookup and its gradient, dropout, 8-bit quantisation and products, and a
run of them together as an encoder uses them.  Tolerances count roundings: half a step of the output's type (eps / 2) for the last
one, 2^-24 for each fp32 operation before it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = {"f32": "float32", "bf16": "bfloat16", "f16": "float16"}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def T():
    import torch
    return torch


@pytest.fixture(scope="module")
def K():
    import paper_2211_12281_b200 as K
    return K


def _gen(T, seed):
    g = T.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _type(T, name):
    return getattr(T, TYPES[name])


def _half_step(T, t):
    return T.finfo(t).eps / 2


def _check(T, got, want, tol, what=""):
    """|got - want| <= tol + the last rounding, element by element; `want` and `tol` in 64 bits."""
    least = T.finfo(got.dtype).smallest_normal * T.finfo(got.dtype).eps / 2        # half the distance of subnormal values
    bound = tol + (want.abs() + tol) * _half_step(T, got.dtype) + least
    diff = (got.double() - want).abs()
    bad = ~(diff <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(diff[bad].max()), bad.nonzero()[:4].tolist())


def _strided(T, rows, cols, dtype, extra=0, shift=0):
    """A matrix whose rows lie cols + extra elements apart and begin `shift` elements into their storage."""
    flat = T.zeros(rows * (cols + extra) + shift, dtype=dtype, device="cuda")
    return flat[shift:].view(rows, cols + extra)[:, :cols]


# ---- lookup ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,E,d,tt,to,scale,extra,shift", [
    (1, 1, 1, "f32", "f32", 1.0, 0, 0), (1, 1000, 256, "bf16", "bf16", 16.0, 0, 0), (5, 7, 5, "f32", "bf16", 0.3, 0, 0),
    (33, 100, 8, "bf16", "f32", 1.0, 0, 0), (1000, 50, 200, "f16", "f16", -2.5, 0, 0), (257, 300, 33, "f16", "f32", 1.7, 3, 1),
    (64, 300, 64, "f32", "f32", 1.0, 4, 0), (64, 300, 64, "f32", "f32", 1.0, 0, 1), (4097, 900, 128, "f32", "f16", 0.125, 0, 0),
    (77, 9, 4096, "bf16", "bf16", 1.0, 8, 0), (3000, 70, 45, "bf16", "f16", 2.0, 0, 0), (100, 70, 46, "f32", "bf16", 2.0, 1, 1), (9, 70, 3, "f16", "f32", 2.0, 0, 0), (3, 9, 1000, "bf16", "f16", 3.0, 0, 2), (24_576, 5000, 20, "f32", "f32", 4.472, 0, 0)])
def test_lookup(T, K, n, E, d, tt, to, scale, extra, shift):
    g = _gen(T, n + d)
    table = _strided(T, E, d, _type(T, tt), extra, shift)
    table.copy_(T.randn((E, d), generator=g, device="cuda"))
    ids = T.randint(0, E, (n,), generator=g, device="cuda", dtype=T.int32)
    out = _strided(T, n, d, _type(T, to), extra, shift)
    guard = out.as_strided((n, d + extra), (d + extra, 1), out.storage_offset()) if extra else None
    if extra:
        guard[:, d:] = 7.0
    status = T.zeros(1, dtype=T.int32, device="cuda")
    K.embedding_lookup(table, ids, out, scale=scale, status=status)
    s32 = float(np.float32(scale))
    _check(T, out, table.double()[ids.long()] * s32, (table.double()[ids.long()] * s32).abs() * U)
    assert status.item() == 0
    if extra:
        assert (guard[:, d:] == 7.0).all()          # what lies between the rows stays


@pytest.mark.parametrize("tt,to", [("bf16", "f16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("n,d", [(1, 1), (999, 1), (85, 45), (86, 45), (3000, 45), (5, 1021), (3, 4095), (2, 4097), (2, 9001)])
@pytest.mark.parametrize("shift", [8, 9, 11, 15])
def test_lookup_of_odd_widths_leaves_its_neighbours(T, K, tt, to, n, d, shift):
    g = _gen(T, n * d + shift)
    table = T.randn((70, d), generator=g, device="cuda").to(_type(T, tt))
    ids = T.randint(-1, 70, (n,), generator=g, device="cuda", dtype=T.int32)
    around = T.full((n * d + shift + 17,), 7.0, device="cuda", dtype=_type(T, to))
    K.embedding_lookup(table, ids, around[shift:shift + n * d].view(n, d), scale=0.5)
    want = T.where(ids[:, None] < 0, T.zeros((), device="cuda"), table[ids.clamp(min=0).long()].float() * 0.5).to(_type(T, to))
    assert T.equal(around[shift:shift + n * d].view(n, d), want)          # half of a value is exact, then one rounding on both sides
    assert (around[:shift] == 7.0).all() and (around[shift + n * d:] == 7.0).all()


def test_lookup_padding_and_bad_ids(T, K):
    table = T.full((10, 24), float("nan"), device="cuda")
    table[2:5] = 1.5
    ids = T.tensor([2, -1, 4, 7, 3], dtype=T.int32, device="cuda")
    out = T.full((5, 24), 9.0, device="cuda")
    status = T.zeros(1, dtype=T.int32, device="cuda")
    K.embedding_lookup(table, ids, out, scale=2.0, padding_id=7, status=status)       # -1 is now an id outside the table
    assert (out[[0, 2, 4]] == 3.0).all() and (out[[1, 3]] == 0.0).all() and status.item() == -8
    status.zero_()
    K.embedding_lookup(table, ids, out, scale=float("inf"), status=status)            # default: -1 is padding, zero whatever the scale
    assert (out[1] == 0.0).all() and status.item() == 0 and T.isnan(out[3]).all() and T.isinf(out[0]).all()
    ids[0], ids[2] = 10, -2147483648
    K.embedding_lookup(table, ids, out, scale=2.0)                                    # no status word: still a zero row
    assert (out[[0, 1, 2]] == 0.0).all()
    K.embedding_lookup(table, ids[:0], out[:0])


def test_rows_beyond_two_to_the_31_elements(T, K):
    E, d = 8_500_000, 256
    table = T.empty((E, d), dtype=T.bfloat16, device="cuda")
    for r in (0, 8_388_607, 8_388_608, E - 1):
        table[r] = T.arange(d, device="cuda") + r % 7
    ids = T.tensor([E - 1, 0, 8_388_608, 8_388_607], dtype=T.int32, device="cuda")
    out = T.empty((4, d), device="cuda")
    K.embedding_lookup(table, ids, out)
    assert (out == table[ids.long()].float()).all()
    grads = T.randn((4, d), device="cuda")
    K.embedding_grad(ids, grads, table)
    assert (table[ids.long()] == grads.to(T.bfloat16)).all()
    assert int((table.view(T.int16).view(E, d) != 0).any(1).sum()) == 4


# ---- gradient --------------------------------------------------------------------------------------------------------

def _id_list(T, g, kind, n, E):
    if kind == "one":
        return T.full((n,), E // 2, dtype=T.int32, device="cuda")
    if kind == "distinct":
        return T.randperm(E, generator=g, device="cuda")[:n].to(T.int32)
    if kind == "blocks":       # runs of every length around the chunks the gradient walks in
        lens = [1, 7, 8, 9, 15, 16, 17, 23, 24, 25, 31, 32, 33, 47, 63, 64, 65, 95, 96, 97, 128, 3, 2, 250, 511, 5]
        ids, at = [], 0
        while len(ids) < n:
            ids += [at % E] * lens[at % len(lens)]
            at += 1
        ids = T.tensor(ids[:n], dtype=T.int32, device="cuda")
        return ids[T.randperm(n, generator=g, device="cuda")]
    u = T.rand(n, generator=g, device="cuda", dtype=T.float64)
    ids = (T.exp(u * float(np.log(E + 1.0))).long() - 1).clamp_(0, E - 1).to(T.int32)
    if kind == "padded":
        ids = T.where(T.rand(n, generator=g, device="cuda") < 0.3, T.full_like(ids, -1), ids)
    return ids


@pytest.mark.parametrize("n,E,d,kind,tg,to,scale,acc", [
    (1, 1, 1, "one", "f32", "f32", 1.0, False), (1, 1000, 32, "zipf", "f32", "f32", 2.0, True), (7, 3, 5, "zipf", "bf16", "f32", 0.5, False),
    (33, 50, 8, "padded", "f16", "f16", 1.0, False), (256, 1000, 32, "zipf", "f32", "f32", 1.0, False), (256, 1000, 32, "one", "f32", "bf16", 1.0, True),
    (1000, 100_000, 64, "distinct", "bf16", "bf16", 1.0, False), (1025, 77, 100, "blocks", "f32", "f32", -1.5, True),
    (2048, 5, 24, "zipf", "f32", "f32", 1.0, False), (2048, 8192, 40, "one", "f32", "f32", 1.0, False), (2047, 70_001, 33, "blocks", "bf16", "bf16", 0.5, True),
    (2000, 900_000, 9, "padded", "f32", "f16", 1.0, False), (30_000, 255, 141, "zipf", "bf16", "bf16", 1.0, False), (150_000, 255, 15, "blocks", "f16", "f32", 1.0, True), (2049, 4000, 200, "blocks", "bf16", "f32", 1.0, False), (2049, 2100, 8, "distinct", "f32", "f32", 1.0, False),
    (5000, 300, 33, "blocks", "f16", "f32", 1.0, False), (5000, 1, 260, "one", "f32", "f32", 0.01, False), (24_576, 100_000, 128, "zipf", "f32", "f32", 1.0, False),
    (24_576, 3000, 520, "padded", "bf16", "f16", 0.01, True), (40_000, 70_000, 7, "blocks", "f32", "f32", 1.0, False),
    (131_071, 999, 16, "blocks", "bf16", "f32", 1.0, False), (131_072, 1000, 16, "blocks", "bf16", "f32", 1.0, False),
    (200_000, 2_100_000, 12, "zipf", "f32", "f32", 1.0, True), (300_000, 5000, 36, "one", "bf16", "f32", 1.0, False),
    (600_000, 120_001, 4, "blocks", "f32", "f32", 1.0, False), (700_003, 4_300_000, 8, "padded", "f16", "f32", 1.0, False)])
def test_grad(T, K, n, E, d, kind, tg, to, scale, acc):
    g = _gen(T, n + d)
    ids = _id_list(T, g, kind, n, E)
    grads = T.randn((n, d), generator=g, device="cuda").to(_type(T, tg))
    old = T.randn((E, d), generator=g, device="cuda").to(_type(T, to))
    status = T.zeros(1, dtype=T.int32, device="cuda")
    runs = []
    for _ in range(2):
        out = old.clone() if acc else T.full_like(old, float("nan"))
        K.embedding_grad(ids, grads, out, scale=scale, accumulate=acc, status=status)
        runs.append(out)
    assert status.item() == 0 and T.equal(runs[0].view(T.uint8), runs[1].view(T.uint8))      # the same bits every time
    keep = ids >= 0
    where = ids[keep].long()
    zeros = lambda: T.zeros((E, d), dtype=T.float64, device="cuda")
    total, size = zeros().index_add_(0, where, grads[keep].double()), zeros().index_add_(0, where, grads[keep].double().abs())
    count = T.bincount(where, minlength=E).double()[:, None]
    s32 = float(np.float32(scale))
    want = total * s32 + (old.double() if acc else 0)
    # every addition of an id's `count` rows rounds once, then the product with the scale and the addition to the old value
    tol = (count * size * abs(s32) + 2 * (size * abs(s32) + (old.double().abs() if acc else 0))) * U
    _check(T, runs[0], want, tol, kind)
    if acc:
        assert T.equal(runs[0][count[:, 0] == 0], old[count[:, 0] == 0])
    else:
        assert (runs[0][count[:, 0] == 0] == 0).all()


@pytest.mark.parametrize("n", [40, 3000, 140_000])
@pytest.mark.parametrize("E,d", [(61, 24), (700, 3), (90, 70), (40, 515)])
def test_grad_of_strided_and_shifted_rows(T, K, n, E, d):
    g = _gen(T, n)
    ids = _id_list(T, g, "zipf", n, E)
    for extra, shift, to in ((8, 0, T.float32), (3, 0, T.float32), (0, 1, T.float32), (4, 2, T.float32), (0, 3, T.bfloat16), (5, 1, T.float16)):
        grads, out = _strided(T, n, d, T.bfloat16, extra, shift), _strided(T, E, d, to, extra, shift)
        grads.copy_(T.randn((n, d), generator=g, device="cuda"))
        all_of = out.as_strided((E, d + extra), (d + extra, 1), out.storage_offset()) if extra else None
        if extra:
            all_of[:-1, d:] = 5.0
        out.fill_(3.0)
        K.embedding_grad(ids, grads, out)
        plain = T.full((E, d), 3.0, device="cuda", dtype=to)
        K.embedding_grad(ids, grads.contiguous(), plain)
        assert T.equal(out, plain)                   # where the rows lie changes nothing
        if extra:
            assert (all_of[:-1, d:] == 5.0).all()


@pytest.mark.parametrize("n", [64, 5000, 140_000])
def test_grad_keeps_bad_and_padded_rows_out(T, K, n):
    g = _gen(T, n)
    E, d = 40, 16
    ids = _id_list(T, g, "zipf", n, E)
    grads = T.randn((n, d), generator=g, device="cuda")
    clean, status = T.empty((E, d), device="cuda"), T.zeros(1, dtype=T.int32, device="cuda")
    some = T.rand(n, generator=g, device="cuda") < 0.2
    some[0] = True
    K.embedding_grad(T.where(some, T.full_like(ids, -1), ids), grads, clean, status=status)
    assert status.item() == 0
    for bad in (E, 2147483647, -2147483648, -7):
        dirty, out = T.where(some, T.full_like(ids, bad), ids), T.empty((E, d), device="cuda")
        spoiled = T.where(some[:, None], T.full_like(grads, float("nan")), grads)
        K.embedding_grad(dirty, spoiled, out, status=status)
        assert status.item() == -8 and T.equal(out, clean)
        status.zero_()
        K.embedding_grad(dirty, spoiled, out, padding_id=bad, status=status)
        assert status.item() == 0 and T.equal(out, clean)
    # a NaN stays with its id
    grads[n // 2] = float("nan")
    K.embedding_grad(ids, grads, clean)
    hit = T.zeros(E, dtype=T.bool, device="cuda")
    hit[ids[n // 2].long()] = True
    assert T.isnan(clean[hit]).all() and T.isfinite(clean[~hit]).all()


def test_grad_of_nothing(T, K):
    out = T.ones((5, 6), device="cuda")
    none = T.empty(0, dtype=T.int32, device="cuda")
    K.embedding_grad(none, T.empty((0, 6), device="cuda"), out, accumulate=True)
    assert (out == 1).all()
    wide = T.ones((5, 9), device="cuda")
    K.embedding_grad(none, T.empty((0, 6), device="cuda"), wide[:, :6])
    assert (wide[:, :6] == 0).all() and (wide[:, 6:] == 1).all()
    out.fill_(1)
    K.embedding_grad(T.full((9,), -1, dtype=T.int32, device="cuda"), T.ones((9, 6), device="cuda"), out)
    assert (out == 0).all()


def test_lookup_and_grad_are_each_others_transpose(T, K):
    """<g, lookup(T)> = <grad(g), T>, and differences of a scalar of the rows."""
    g = _gen(T, 3)
    n, E, d, scale = 300, 90, 20, 1.25
    ids = _id_list(T, g, "padded", n, E)
    table, grads = T.randn((E, d), generator=g, device="cuda"), T.randn((n, d), generator=g, device="cuda")
    rows, dt = T.empty((n, d), device="cuda"), T.empty((E, d), device="cuda")
    K.embedding_lookup(table, ids, rows, scale=scale)
    K.embedding_grad(ids, grads, dt, scale=scale)
    left, right = (grads.double() * rows.double()).sum(), (dt.double() * table.double()).sum()
    assert abs(left - right) <= 20 * U * (grads.double() * rows.double()).abs().sum()
    e, k, step = int(ids[ids >= 0][0]), 4, 2.0 ** -4            # the map is linear: a difference is exact up to roundings
    moved = table.clone()
    moved[e, k] += step
    rows2 = T.empty_like(rows)
    K.embedding_lookup(moved, ids, rows2, scale=scale)
    slope = (grads.double() * (rows2.double() - rows.double())).sum() / (moved[e, k].double() - table[e, k].double())
    assert abs(slope - dt[e, k].double()) <= 64 * U / step * (grads.double().abs() * rows.double().abs())[ids == e].sum() + 1e-5


# ---- dropout ---------------------------------------------------------------------------------------------------------

def _philox_halves(n, seed, step, site):
    """The documented 16-bit numbers, from the generator's definition."""
    x = [np.arange((n + 7) // 8, dtype=np.uint64)] + [np.full((n + 7) // 8, v, dtype=np.uint64) for v in (step & 0xFFFFFFFF, step >> 32, (1 << 31) + site)]
    k0, k1, low, m = seed & 0xFFFFFFFF, seed >> 32, np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> m) ^ x[1] ^ np.uint64(k0), q & low, (p >> m) ^ x[3] ^ np.uint64(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack([h for w in x for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 1).reshape(-1)[:n]


@pytest.mark.parametrize("n,p,tx,to,res,shift", [
    (1, 0.5, "f32", "f32", False, 0), (7, 0.5, "bf16", "bf16", True, 0), (8, 0.1, "f16", "f16", False, 0), (9, 0.25, "f32", "bf16", True, 0),
    (2048, 0.0, "f32", "f32", True, 0), (2049, 1.0, "bf16", "f32", False, 0), (100_003, 0.1, "f32", "f32", False, 0), (100_003, 0.1, "bf16", "bf16", True, 1),
    (65_536, 0.3, "f16", "f32", True, 3), (65_536, 1e-6, "f32", "f16", False, 0), (1_000_000, 0.9, "bf16", "f16", False, 0)])
def test_dropout(T, K, n, p, tx, to, res, shift):
    g = _gen(T, n)
    x = T.randn(n + shift, generator=g, device="cuda").to(_type(T, tx))[shift:]
    r = T.randn(n + shift, generator=g, device="cuda").to(_type(T, to))[shift:] if res else None
    seed, step, site = 0x123456789ABCDEF0 + n, (5 << 32) + 17, 41
    out = T.full((n + shift,), 3.0, device="cuda", dtype=_type(T, to))[shift:]
    K.dropout(x, out, p, seed, step, site=site, residual=r)
    cut = round(p * 65536)
    keep = T.from_numpy((_philox_halves(n, seed, step, site) >= cut)).cuda()
    y = x.double() * (65536 / (65536 - cut) if cut < 65536 else 0.0)
    want = T.where(keep, y, T.zeros_like(y)) + (r.double() if res else 0)
    _check(T, out, want, 2 * U * y.abs() + U * want.abs())
    if not res:
        assert (out[~keep] == 0).all()
    # in place: on x, and on the residual
    if tx == to:
        xx = x.clone()
        K.dropout(xx, xx, p, seed, step, site=site, residual=r)
        assert T.equal(xx, out)
    if res:
        rr = r.clone()
        K.dropout(x, rr, p, seed, step, site=site, residual=rr)
        assert T.equal(rr, out)


def test_dropout_masks_differ_by_seed_step_and_site_and_drop_infinities(T, K):
    n = 40_000
    x, masks = T.full((n,), float("inf"), device="cuda"), []
    for seed, step, site in ((1, 0, 0), (2, 0, 0), (1 << 32, 0, 0), (1, 1, 0), (1, 1 << 32, 0), (1, 0, 1)):
        out = T.empty_like(x)
        K.dropout(x, out, 0.5, seed, step, site=site)
        assert ((out == 0) | T.isinf(out)).all()
        masks.append(out == 0)
    for i in range(len(masks)):
        assert abs(int(masks[i].sum()) - n // 2) < 6 * (n / 4) ** 0.5        # six standard deviations
        for j in range(i):
            assert abs(int((masks[i] == masks[j]).sum()) - n // 2) < 6 * (n / 4) ** 0.5


def test_dropout_backward_is_the_same_call(T, K):
    g = _gen(T, 9)
    x, dy = (T.randn(5000, generator=g, device="cuda") for _ in range(2))
    y, dx = T.empty_like(x), T.empty_like(x)
    K.dropout(x, y, 0.2, 77, 3, site=2)
    K.dropout(dy, dx, 0.2, 77, 3, site=2)
    left, right = (dy.double() * y.double()).sum(), (dx.double() * x.double()).sum()
    assert abs(left - right) <= 8 * U * (dy.double() * y.double()).abs().sum()
    assert T.equal(dx == 0, y == 0)


def test_dropout_in_a_graph_draws_a_new_mask_at_every_replay(T, K):
    n = 4096
    x, out, step = T.ones(n, device="cuda"), T.empty(n, device="cuda"), T.zeros(1, dtype=T.int64, device="cuda")
    side = T.cuda.Stream()
    side.wait_stream(T.cuda.current_stream())
    with T.cuda.stream(side):
        K.dropout(x, out, 0.5, 5, 100, step_dev=step)
    T.cuda.current_stream().wait_stream(side)
    graph = T.cuda.CUDAGraph()
    with T.cuda.graph(graph):
        K.dropout(x, out, 0.5, 5, 100, step_dev=step)
        step.add_(1)
    for k in range(3):
        graph.replay()
        want = T.empty_like(x)
        K.dropout(x, want, 0.5, 5, 100 + k)
        assert T.equal(out, want)
    assert step.item() == 3


# ---- 8-bit quantisation ----------------------------------------------------------------------------------------------

FP8 = {"e4m3": ("float8_e4m3fn", 448.0, 3, -6), "e5m2": ("float8_e5m2", 57344.0, 2, -14)}


def _empty8(T, rows, cols, fmt, ld_extra=0):
    return T.zeros((rows, (cols + 15) // 16 * 16 + ld_extra), dtype=T.uint8, device="cuda").view(getattr(T, FP8[fmt][0]))[:, :cols]


def _quantized(T, x, fmt, block, pow2):
    """(8-bit values in 64 bits, scales [blocks of K, rows or blocks of rows]) by the definition; finite x only."""
    _, top, bits, least = FP8[fmt]
    rows, cols = x.shape
    x = x.double()
    pad = T.nn.functional.pad(x.abs(), (0, -cols % 128, 0, -rows % block))
    most = pad.reshape(pad.shape[0] // block, block, -1, 128).amax(3).amax(1)
    s = (most.float() / T.full_like(most, top, dtype=T.float32)).clamp(min=2.0 ** -126)
    if pow2:
        m, e = T.frexp(s)
        s = T.ldexp(T.ones_like(s), e - (m == 0.5).int())
    s = T.where(most > 0, s, T.ones_like(s))
    y = x / s.double().repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    step = T.exp2((T.frexp(y)[1] - 1).clamp(min=least).double() - bits)
    return T.round(y / step) * step, s.t().contiguous()


def _codes(T, q):
    return q.contiguous().view(T.uint8)


@pytest.mark.parametrize("rows,cols,tx,fmt,block,pow2,extra,shift", [
    (1, 1, "f32", "e4m3", 1, False, 0, 0), (1, 768, "bf16", "e4m3", 1, False, 0, 0), (3, 130, "f32", "e5m2", 1, False, 0, 0),
    (128, 128, "bf16", "e4m3", 128, False, 0, 0), (200, 300, "f16", "e4m3", 1, True, 0, 0), (257, 768, "f32", "e4m3", 1, False, 5, 1),
    (257, 520, "bf16", "e5m2", 128, True, 8, 0), (1000, 64, "f32", "e4m3", 128, False, 0, 0), (130, 1000, "bf16", "e4m3", 1, False, 1, 0),
    (4100, 256, "f32", "e5m2", 1, True, 0, 0), (2500, 384, "f16", "e5m2", 1, False, 0, 0), (700, 24, "bf16", "e4m3", 128, False, 0, 4)])
def test_quantize(T, K, rows, cols, tx, fmt, block, pow2, extra, shift):
    g = _gen(T, rows + cols)
    x = _strided(T, rows, cols, _type(T, tx), extra, shift)
    x.copy_(T.randn((rows, cols), generator=g, device="cuda") * T.exp(2 * T.randn((rows, 1), generator=g, device="cuda")))
    if rows > 2:
        x[rows // 2] = 0                                                       # a row of zeros
        x[rows // 3] = x[rows // 3] * 2.0 ** -8                                # values below the type's normal range
    want, ws = _quantized(T, x, fmt, block, pow2)
    want_t, wst = _quantized(T, x.t(), fmt, block, pow2)
    shape = lambda r, c: ((c + 127) // 128, r if block == 1 else (r + 127) // 128)
    q, s = _empty8(T, rows, cols, fmt, 16), T.full(shape(rows, cols), -1.0, device="cuda")
    qt, st = _empty8(T, cols, rows, fmt), T.full(shape(cols, rows), -1.0, device="cuda")
    K.fp8_quantize(x, q, s, qt, st, block_rows=block, pow2=pow2)
    for got, sc, w, wsc in ((q, s, want, ws), (qt, st, want_t, wst)):
        assert T.equal(sc, wsc)
        assert T.equal(got.float().double(), w), int((got.float().double() != w).sum())
    ld = q.stride(0)
    assert (q.view(T.uint8).as_strided((rows, ld), (ld, 1))[:-1, cols:] == 0).all()           # between the rows nothing is written
    q1, s1 = _empty8(T, rows, cols, fmt), T.empty_like(s)
    K.fp8_quantize(x, q1, s1, block_rows=block, pow2=pow2)
    q2, s2 = _empty8(T, cols, rows, fmt), T.empty_like(st)
    K.fp8_quantize(x, qt=q2, scales_t=s2, block_rows=block, pow2=pow2)
    assert T.equal(_codes(T, q1), _codes(T, q)) and T.equal(s1, s) and T.equal(_codes(T, q2), _codes(T, qt)) and T.equal(s2, st)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantize_rounds_the_true_quotient(T, K, fmt):
    """Values on, and one step beside, the middle of two 8-bit values times scales of every kind."""
    _, top, bits, least = FP8[fmt]
    g = _gen(T, 4)
    rows, cols = 4096, 128
    scale = T.exp(3 * T.randn((rows, 1), generator=g, device="cuda", dtype=T.float64)).float().double()
    e = T.randint(least - 3, 8 if fmt == "e4m3" else 15, (rows, cols), generator=g, device="cuda").double()
    k = T.randint(0, 1 << (bits + 1), (rows, cols), generator=g, device="cuda").double()
    mid = ((1 << (bits + 1)) + k) * T.exp2(e - bits - 1)                       # every second one is a middle
    x = (mid.clamp(max=top) * scale).float()
    x = T.where(T.rand((rows, cols), generator=g, device="cuda") < 0.5, x, T.nextafter(x, T.full_like(x, float("inf"))))
    x[:, 0] = (top * scale[:, 0]).float()
    want, ws = _quantized(T, x, fmt, 1, False)
    q, s = _empty8(T, rows, cols, fmt), T.empty((1, rows), device="cuda")
    K.fp8_quantize(x, q, s)
    assert T.equal(s, ws) and T.equal(q.float().double(), want), int((q.float().double() != want).sum())


@pytest.mark.parametrize("tx,fmt,block", [("bf16", "e4m3", 1), ("bf16", "e5m2", 1), ("f16", "e4m3", 1), ("f16", "e5m2", 1), ("bf16", "e4m3", 128), ("f16", "e5m2", 128)])
def test_quantize_rounds_the_true_quotient_of_16_bit_values(T, K, tx, fmt, block):
    """Every mantissa of a block's largest value against a spread of the others' mantissas and exponents: with 16-bit values the
    quotient falls on the middle of two 8-bit values, or a rounding of the scale beside it, two times in a thousand."""
    bits = 7 if tx == "bf16" else 10
    rows, cols = (1 << bits), 128
    top = (1 + T.arange(rows, device="cuda").double() / rows) * 2.0 ** -2
    if block == 128:
        rows = min(rows, 512)
        top = top[:: len(top) // rows].repeat_interleave(128)[: 128 * rows]          # one largest value per block of 128 rows
    g = _gen(T, 6)
    n = top.numel()
    mant = 1 + T.randint(0, 1 << bits, (n, cols * 8), generator=g, device="cuda").double() / (1 << bits)
    x = mant * T.exp2(-T.randint(0, 12 if tx == "bf16" else 9, mant.shape, generator=g, device="cuda").double())
    x = T.where(x < 1, x, x / 2) * top[:, None]                                      # below the largest value ...
    x = x.to(_type(T, tx))
    x = T.where(x.double() > top[:, None], top[:, None].to(x.dtype), x)
    x[:, ::128] = top[:, None].to(x.dtype)                                           # ... which stands first in every block
    want, ws = _quantized(T, x, fmt, block, False)
    q = _empty8(T, n, cols * 8, fmt)
    s = T.empty((cols * 8 // 128, n if block == 1 else (n + 127) // 128), device="cuda")
    K.fp8_quantize(x, q, s, block_rows=block)
    assert T.equal(s, ws) and T.equal(q.float().double(), want), int((q.float().double() != want).sum())


@pytest.mark.parametrize("block", [1, 128])
def test_quantize_of_extreme_blocks(T, K, block):
    x = T.ones((256, 256), device="cuda")
    x[0, 3], x[140, 130] = float("inf"), float("nan")
    x[1] = 0
    x[130:256, :128] = 1e-44
    x[130:256, :128][1:] = 3e38
    q, s = _empty8(T, 256, 256, "e4m3"), T.empty((2, 256 if block == 1 else 2), device="cuda")
    K.fp8_quantize(x, q, s, block_rows=block)
    spread = s.t() if block == 1 else s.t().repeat_interleave(128, 0)
    got = q.float() * spread.repeat_interleave(128, 1)
    bad = T.zeros((256, 256), dtype=T.bool, device="cuda")
    if block == 1:
        bad[0, :128], bad[140, 128:] = True, True
    else:
        bad[:128, :128], bad[128:, 128:] = True, True
    assert T.isnan(got[bad]).all() and T.isfinite(got[~bad]).all()
    assert (got[1][~bad[1]] == 0).all()
    # each of the others is off by at most half a step of a value whose block's largest is 448 steps of scale, or half the smallest step
    off = (got - x)[~bad].abs().double()
    least = spread.repeat_interleave(128, 1)[~bad].double() * 2.0 ** -10
    assert (off <= T.maximum(x[~bad].abs().double() * 2.0 ** -4, least) * (1 + 1e-6)).all()


# ---- 8-bit product ---------------------------------------------------------------------------------------------------

def _operand(T, K, g, rows, k, fmt, block, spread=1.0):
    x = T.randn((rows, k), generator=g, device="cuda") * T.exp(spread * T.randn((rows, 1), generator=g, device="cuda"))
    q = _empty8(T, rows, k, fmt)
    s = T.empty(((k + 127) // 128, rows if block == 1 else (rows + 127) // 128), device="cuda")
    K.fp8_quantize(x, q, s, block_rows=block)
    return q, s


def _stands_for(T, q, s):
    rows, k = q.shape
    s = s if s.shape[1] == rows else s.repeat_interleave(128, 1)[:, :rows]
    return q.float().double() * s.double().repeat_interleave(128, 0)[:k].t()


def _product_tol(T, a, b, k):
    """A block's 128 products (exact in fp32) are added by the tensor cores, each addition off by at most one unit of its 24 bits;
    the product of the scales, its product with the sum and the addition round once each, per block."""
    return (128 * 2 * U + ((k + 127) // 128 + 2) * U) * (a.abs() @ b.abs().t())


@pytest.mark.parametrize("M,N,Kd,fa,fb,ba,bb,to,add", [
    (1, 1, 1, "e4m3", "e4m3", 1, 1, "f32", False), (1, 16, 32, "e4m3", "e4m3", 1, 128, "f32", False), (1, 256, 768, "e4m3", "e4m3", 1, 128, "bf16", False),
    (7, 33, 100, "e4m3", "e5m2", 1, 1, "f32", True), (128, 128, 128, "e5m2", "e4m3", 128, 128, "f16", False), (130, 257, 300, "e4m3", "e4m3", 1, 128, "f32", True),
    (129, 130, 129, "e5m2", "e5m2", 128, 1, "bf16", True), (300, 1000, 1000, "e4m3", "e4m3", 1, 1, "f32", False), (513, 384, 2048, "e4m3", "e4m3", 128, 128, "f32", True),
    (2000, 256, 768, "e4m3", "e4m3", 1, 128, "f32", True), (256, 768, 24_576, "e4m3", "e4m3", 1, 1, "f32", True), (40, 64, 70_000, "e5m2", "e4m3", 1, 1, "f32", False),
    (3, 5000, 4000, "e4m3", "e4m3", 1, 128, "f16", False), (5000, 3, 515, "e4m3", "e4m3", 1, 128, "f32", False), (20_000, 640, 256, "e4m3", "e4m3", 1, 1, "bf16", False),
    (3000, 2502, 125, "e4m3", "e4m3", 1, 128, "bf16", True), (3000, 2501, 130, "e5m2", "e4m3", 1, 1, "f16", True), (3000, 2503, 200, "e4m3", "e4m3", 1, 128, "f32", True),
    (30_000, 60, 300, "e4m3", "e4m3", 1, 128, "f32", True), (30_000, 200, 300, "e4m3", "e4m3", 128, 1, "bf16", True), (2600, 2051, 2300, "e4m3", "e4m3", 1, 128, "bf16", True),
    (2600, 2053, 2300, "e4m3", "e4m3", 1, 1, "f32", False), (2600, 2048, 2300, "e4m3", "e4m3", 1, 128, "f32", True), (2600, 2048, 2300, "e5m2", "e4m3", 128, 1, "bf16", False),
    (4096, 2816, 2049, "e4m3", "e4m3", 1, 1, "f16", True), (120, 38_000, 2100, "e4m3", "e4m3", 1, 128, "bf16", False), (120, 38_000, 2100, "e4m3", "e4m3", 1, 1, "f32", True),
    (130, 700, 2050, "e4m3", "e4m3", 1, 128, "f32", True), (500, 760, 4000, "e4m3", "e5m2", 1, 1, "bf16", True), (1000, 1100, 4100, "e4m3", "e4m3", 1, 128, "f32", False),
    (250, 900, 1030, "e4m3", "e4m3", 128, 128, "f16", True), (17, 4000, 900, "e4m3", "e4m3", 1, 128, "bf16", False), (2, 300, 260, "e5m2", "e4m3", 1, 1, "f32", True)])
def test_product(T, K, M, N, Kd, fa, fb, ba, bb, to, add):
    g = _gen(T, M + N + Kd)
    a, sa = _operand(T, K, g, M, Kd, fa, ba)
    b, sb = _operand(T, K, g, N, Kd, fb, bb, 0.3)
    if to == "f16":
        sa.mul_(2.0 ** -10)                       # sums well inside the type's range
    c0 = T.randn((M, N), generator=g, device="cuda").to(_type(T, to)) if add else None
    va, vb = _stands_for(T, a, sa), _stands_for(T, b, sb)
    want, tol = va @ vb.t(), _product_tol(T, va, vb, Kd)
    if add:
        want = want + c0.double()
        tol = tol + U * want.abs()
    status = T.zeros(1, dtype=T.int32, device="cuda")
    outs = []
    for extra, shift in ((0, 0), (3, 1)):
        out = _strided(T, M, N, _type(T, to), extra, shift)
        out.fill_(float("nan"))
        K.fp8_matmul(a, sa, b, sb, out, addend=c0, status=status)
        outs.append(out)
    assert status.item() == 0
    _check(T, outs[0], want, tol)
    assert T.equal(outs[0], outs[1])              # where the rows of out lie changes nothing
    if add:                                       # onto what out holds
        out = c0.clone()
        K.fp8_matmul(a, sa, b, sb, out, addend=out)
        assert T.equal(out, outs[0])


def test_product_keeps_nan_with_its_row_and_column(T, K):
    g = _gen(T, 8)
    x, w = T.randn((300, 400), generator=g, device="cuda"), T.randn((270, 400), generator=g, device="cuda")
    x[131, 390], w[7, 3] = float("nan"), float("inf")
    a, sa, b, sb = _empty8(T, 300, 400, "e4m3"), T.empty((4, 300), device="cuda"), _empty8(T, 270, 400, "e4m3"), T.empty((4, 270), device="cuda")
    K.fp8_quantize(x, a, sa)
    K.fp8_quantize(w, b, sb)
    out = T.zeros((300, 270), device="cuda")
    K.fp8_matmul(a, sa, b, sb, out)
    bad = T.zeros((300, 270), dtype=T.bool, device="cuda")
    bad[131], bad[:, 7] = True, True
    assert T.isnan(out[bad]).all() and T.isfinite(out[~bad]).all()


def test_product_reads_nothing_beyond_its_columns(T, K):
    """Bytes between a row's last column and the next row may hold anything (here NaN)."""
    g = _gen(T, 12)
    a, sa = _operand(T, K, g, 200, 300, "e4m3", 1)
    b, sb = _operand(T, K, g, 140, 300, "e4m3", 1)
    want = T.empty((200, 140), device="cuda")
    K.fp8_matmul(a, sa, b, sb, want)
    for q in (a, b):
        ld = q.stride(0)
        q.view(T.uint8).as_strided((q.shape[0], ld), (ld, 1))[:, 300:] = 0x7F
    out = T.empty_like(want)
    K.fp8_matmul(a, sa, b, sb, out)
    assert T.equal(out, want)


# ---- as they are used ------------------------------------------------------------------------------------------------

def _encoder(T, K, case, table, feat, matrix, ids, dz, seed, step):
    """z = dropout(scale table[ids] + M features) and the gradients of table and M, all by the library."""
    n, d, F, scale, p = case["n"], case["d"], case["F"], 0.5, 0.25
    rows, z, dpre, dt = (T.empty(s, device="cuda") for s in ((n, d), (n, d), (n, d), tuple(table.shape)))
    fq, fs, ft, fts = _empty8(T, n, F, "e4m3"), T.empty(((F + 127) // 128, n), device="cuda"), _empty8(T, F, n, "e4m3"), T.empty(((n + 127) // 128, F), device="cuda")
    mq, ms = _empty8(T, d, F, "e4m3"), T.empty(((F + 127) // 128, (d + 127) // 128), device="cuda")
    gt, gts = _empty8(T, d, n, "e5m2"), T.empty(((n + 127) // 128, d), device="cuda")
    dm = T.empty((d, F), device="cuda")

    def forward_backward():
        K.embedding_lookup(table, ids, rows, scale=scale)
        K.fp8_quantize(feat, fq, fs, ft, fts)
        K.fp8_quantize(matrix, mq, ms, block_rows=128)
        K.fp8_matmul(fq, fs, mq, ms, rows, addend=rows)
        K.dropout(rows, z, p, seed, step)
        K.dropout(dz, dpre, p, seed, step)
        K.embedding_grad(ids, dpre, dt, scale=scale)
        K.fp8_quantize(dpre, qt=gt, scales_t=gts)
        K.fp8_matmul(gt, gts, ft, fts, dm)
    return forward_backward, dict(z=z, dt=dt, dm=dm)


def _encoder_inputs(T, case, seed):
    g = _gen(T, seed)
    n, E, d, F = case["n"], case["E"], case["d"], case["F"]
    return (T.randn((E, d), generator=g, device="cuda"), T.randn((n, F), generator=g, device="cuda").to(T.bfloat16),
            T.randn((d, F), generator=g, device="cuda") * F ** -0.5, _id_list(T, g, "zipf", n, E), T.randn((n, d), generator=g, device="cuda"))


@pytest.mark.parametrize("case", [dict(n=64, E=50, d=32, F=64), dict(n=500, E=300, d=200, F=384), dict(n=3000, E=1000, d=256, F=768)])
def test_encoder_of_rows_and_features(T, K, case):
    table, feat, matrix, ids, dz = _encoder_inputs(T, case, 5)
    call, got = _encoder(T, K, case, table, feat, matrix, ids, dz, 99, 7)
    call()
    # in 64 bits, with the roundings to 8 bits where the path has them
    stand = lambda x, fmt, block: (lambda q, s: q * (s if s.shape[1] == x.shape[0] else s.repeat_interleave(128, 1)[:, :x.shape[0]]).double()
                                   .repeat_interleave(128, 0)[:x.shape[1]].t())(*_quantized(T, x, fmt, block, False))
    keep = T.from_numpy(_philox_halves(dz.numel(), 99, 7, 0) >= 16384).cuda().view_as(dz).double() * (65536 / 49152)
    vf, vm = stand(feat, "e4m3", 1), stand(matrix, "e4m3", 128)
    pre = 0.5 * table.double()[ids.long()] + vf @ vm.t()
    tol = _product_tol(T, vf, vm, case["F"]) + 4 * U * (0.5 * table.double()[ids.long()].abs() + pre.abs())
    _check(T, got["z"], pre * keep, tol * keep + 4 * U * pre.abs())
    dpre = dz.double() * keep
    zeros = lambda: T.zeros_like(table, dtype=T.float64)
    size = zeros().index_add_(0, ids.long(), dpre.abs())
    count = T.bincount(ids.long(), minlength=case["E"]).double()[:, None]
    _check(T, got["dt"], 0.5 * zeros().index_add_(0, ids.long(), dpre), (count + 4) * U * size)
    # the gradient's 8-bit values are taken of dpre in fp32, as the path does
    dpre32 = T.empty_like(dz)
    K.dropout(dz, dpre32, 0.25, 99, 7)
    vg, vt = stand(dpre32.t(), "e5m2", 1), stand(feat.t(), "e4m3", 1)
    _check(T, got["dm"], vg @ vt.t(), _product_tol(T, vg, vt, case["n"]))
    # and the whole gradient is that of the unrounded map up to the 8-bit types' half steps (2^-3 and 2^-4 of a value, or half the
    # smallest step of its block): |dpre|^T |feat| times their sum bounds it, the smallest steps are a 2^-9 of a block's largest at most
    full = dpre.t() @ feat.double()
    bound = (2.0 ** -3 + 2.0 ** -4 + 2.0 ** -7) * (dpre.abs().t() @ feat.double().abs())
    assert ((got["dm"].double() - full).abs() <= bound + 1e-3).all()


@pytest.mark.parametrize("fmt,F,d,opt,own", [("e4m3", 768, 64, "sgd", True), ("e5m2", 192, 40, "adagrad", False), ("e4m3", 64, 32, "adam", True),
                                              ("e4m3", 1088, 72, "sgd", False)])
def test_training_step_on_features_in_8_bits(T, K, fmt, F, d, opt, own):
    """A step on 8-bit features is, bit for bit, the step on the bf16 values that they stand for."""
    from parity_util import GpuSide, Problem
    sides = []
    for eight in (True, False):
        prob = Problem(E=900, R=5, T=9000, d=d, score="distmult", loss="softmax", opt=opt, B=64, N=128, P=2, lr=0.02, graph_seed=29)
        prob.kw.update(feat_dim=F, feat_shared=0)
        gpu = GpuSide(prob)
        g = _gen(T, 3)
        x = T.randn((prob.E, F), generator=g, device="cuda") * T.exp(T.randn((prob.E, 1), generator=g, device="cuda")) * F ** -0.5
        mats = [T.randn((d, F), generator=g, device="cuda").mul_(0.3) for _ in range(2)]
        shape = {"sgd": None, "adam": (d, 2 * F), "adagrad": (d,)}[opt]
        states = [None if shape is None else T.zeros(shape, device="cuda") for _ in range(2)]
        q, s = _empty8(T, prob.E, F, fmt, 16), T.empty(((F + 127) // 128, prob.E), device="cuda")
        K.fp8_quantize(x, q, s)
        if eight:
            gpu.kge.bind_features_fp8(q, s, *mats, *states)
        else:
            gpu.kge.bind_features(_stands_for(T, q, s).to(T.bfloat16), *mats, *states)      # (a product of 4 and 24 bits is exact in 64: one rounding)
        loss = T.zeros(1, device="cuda")
        for step in range(2):
            ids = () if own else [gpu.dev_i32(a) for a in gpu.sample(step)]
            gpu.kge.train_step(step, prob.lr, *ids, loss_out=loss)
        assert gpu.kge.get_status() == 0
        sides.append([gpu.ent, gpu.rel, loss, *mats] + [v for v in states if v is not None])
    for a, b in zip(*sides):
        assert T.isfinite(a).all() and T.equal(a, b)


def test_features_in_8_bits_are_checked(T, K):
    from parity_util import GpuSide, Problem
    prob = Problem(E=90, R=3, T=500, d=32, score="transe", B=4, N=4, P=1)
    prob.kw.update(feat_dim=64)
    gpu = GpuSide(prob)
    mats = [T.zeros((32, 64), device="cuda") for _ in range(2)]
    q, s = _empty8(T, 90, 64, "e4m3"), T.ones((1, 90), device="cuda")
    for feat, scales in ((q[:89], s[:, :89].contiguous()), (q[:, :48], s), (q, T.ones((1, 1), device="cuda"))):
        with pytest.raises(K.KgeError) as e:
            gpu.kge.bind_features_fp8(feat, scales, *mats)
        assert e.value.code == -1
    gpu.kge.bind_features_fp8(q, s, *mats)


def test_captured_runs_replay_beside_eager_ones(T, K):
    """Two captured graphs with scratch of their own on two streams, replayed together, give what eager calls give."""
    cases = [dict(n=3000, E=1000, d=64, F=256), dict(n=2500, E=40, d=64, F=384)]
    made = []
    for i, case in enumerate(cases):
        args = _encoder_inputs(T, case, 20 + i)
        call, got = _encoder(T, K, case, *args, 11 + i, 3)
        call()
        T.cuda.synchronize()
        want = {k: v.clone() for k, v in got.items()}
        graph, stream = T.cuda.CUDAGraph(), T.cuda.Stream()
        with T.cuda.graph(graph, stream=stream):
            call()
        made.append((graph, stream, got, want, call))           # (the call holds the inputs that the graph reads)
    for _ in range(3):
        for graph, stream, got, _, _ in made:
            with T.cuda.stream(stream):
                for v in got.values():
                    v.fill_(float("nan"))
                graph.replay()
        T.cuda.synchronize()
        for _, _, got, want, _ in made:
            for k in want:
                assert T.equal(got[k], want[k]), k


def test_first_calls_of_a_process_can_be_captured():
    """Nothing that a first call sets up (kernel attributes, tensor maps, what the device offers) needs to happen outside a capture."""
    import subprocess
    import sys
    from pathlib import Path
    code = r"""
import torch
import paper_2211_12281_b200 as K
dev = "cuda"
e8 = lambda r, c: torch.empty((r, c), dtype=torch.float8_e4m3fn, device=dev)
ids = torch.arange(5000, dtype=torch.int32, device=dev) % 700
table, rows, dt = torch.randn((700, 64), device=dev), torch.zeros((5000, 64), device=dev), torch.zeros((700, 64), device=dev)
w, wq, ws = torch.randn((128, 64), device=dev), e8(128, 64), torch.empty((1, 1), device=dev)
q, s, y = e8(5000, 64), torch.empty((1, 5000), device=dev), torch.zeros((5000, 128), device=dev)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    K.embedding_lookup(table, ids, rows)
    K.dropout(rows, rows, 0.5, 3)
    K.fp8_quantize(rows, q, s)
    K.fp8_quantize(w, wq, ws, block_rows=128)
    K.fp8_matmul(q, s, wq, ws, y)
    K.embedding_grad(ids, rows, dt)
g.replay()
torch.cuda.synchronize()
a = [t.clone() for t in (rows, y, dt)]
K.embedding_lookup(table, ids, rows)
K.dropout(rows, rows, 0.5, 3)
K.fp8_quantize(rows, q, s)
K.fp8_quantize(w, wq, ws, block_rows=128)
K.fp8_matmul(q, s, wq, ws, y)
K.embedding_grad(ids, rows, dt)
assert all(torch.equal(x, t) for x, t in zip(a, (rows, y, dt))) and float(a[1].abs().sum()) > 0 and float(a[2].abs().sum()) > 0
"""
    res = subprocess.run([sys.executable, "-c", code], cwd=Path(__file__).resolve().parent.parent, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-2000:]


def test_calls_on_nothing(T, K):
    i0 = T.empty(0, dtype=T.int32, device="cuda")
    K.embedding_lookup(T.ones((3, 8), device="cuda"), i0, T.empty((0, 8), device="cuda"))
    K.dropout(T.empty(0, device="cuda"), T.empty(0, device="cuda"), 0.5, 1)
    K.fp8_quantize(T.empty((0, 64), device="cuda"), _empty8(T, 0, 64, "e4m3"), T.empty((1, 0), device="cuda"))
    b, sb = _operand(T, K, _gen(T, 1), 32, 64, "e4m3", 1)
    K.fp8_matmul(_empty8(T, 0, 64, "e4m3"), T.empty((1, 0), device="cuda"), b, sb, T.empty((0, 32), device="cuda"))


def test_scratch_of_the_callers_is_used_and_checked(T, K):
    g = _gen(T, 2)
    n, E, d = 5000, 100, 16
    ids, grads, out = _id_list(T, g, "zipf", n, E), T.randn((n, d), generator=g, device="cuda"), T.empty((E, d), device="cuda")
    need = K.embedding_grad_scratch_bytes(E, d, n)
    want = T.empty_like(out)
    K.embedding_grad(ids, grads, want)
    K.embedding_grad(ids, grads, out, scratch=T.empty(need + 256, dtype=T.uint8, device="cuda"))
    assert T.equal(out, want)
    with pytest.raises(K.KgeError) as e:
        K.embedding_grad(ids, grads, out, scratch=T.empty(need // 2, dtype=T.uint8, device="cuda"))
    assert e.value.code == -4
