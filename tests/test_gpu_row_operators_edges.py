"""The operators on rows where they could go wrong: non-finite values in every input type, sums whose order must not follow the layout,
scales far from one, very wide rows, waits that run out, and arrays beyond 2^31 elements.  Tolerances count roundings: half a step of
the output's type for the last one, 2^-24 for each fp32 operation before it."""
import numpy as np
import pytest

from test_gpu_row_operators import K, T, U, _check, _empty8, _gen, _id_list, _product_tol, _quantized, _stands_for, _strided, _type  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- 8-bit quantisation ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tx", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block,pow2", [(1, False), (1, True), (128, False), (128, True)])
def test_a_block_with_an_infinity_or_a_nan_stands_for_nan(T, K, tx, fmt, block, pow2):
    """Each value of such a block is NaN, the infinity itself too, in both orientations and alone; the other blocks are as without it."""
    g = _gen(T, 17)
    x = T.randn((300, 400), generator=g, device="cuda").to(_type(T, tx))
    clean = x.clone()
    inf = float("inf")
    spots = [(3, 5, inf), (3, 390, -inf), (140, 200, -inf), (141, 201, inf), (299, 399, float("nan")), (260, 130, inf), (260, 131, -inf)]
    for r, c, v in spots:
        x[r, c] = v
    shape = lambda r, c: ((c + 127) // 128, r if block == 1 else (r + 127) // 128)
    q, s = _empty8(T, 300, 400, fmt), T.empty(shape(300, 400), device="cuda")
    qt, st = _empty8(T, 400, 300, fmt), T.empty(shape(400, 300), device="cuda")
    q1, s1 = _empty8(T, 300, 400, fmt), T.empty_like(s)
    K.fp8_quantize(x, q, s, qt, st, block_rows=block, pow2=pow2)
    K.fp8_quantize(x, q1, s1, block_rows=block, pow2=pow2)
    for codes, scales, src, at in ((q, s, clean, spots), (q1, s1, clean, spots), (qt, st, clean.t(), [(c, r, v) for r, c, v in spots])):
        bad = T.zeros(tuple(src.shape), dtype=T.bool, device="cuda")
        for r, c, _ in at:
            r0 = r // block * block
            bad[r0:r0 + block, c // 128 * 128:c // 128 * 128 + 128] = True
        got, (want, ws) = _stands_for(T, codes, scales), _quantized(T, src, fmt, block, pow2)
        assert T.isnan(got[bad]).all(), (int((~T.isnan(got[bad])).sum()), got[bad][~T.isnan(got[bad])][:4])
        assert T.equal(codes.float().double()[~bad], want[~bad]) and T.isfinite(got[~bad]).all()


@pytest.mark.parametrize("tx", ["f32", "bf16", "f16"])
def test_an_infinity_makes_its_rows_products_nan(T, K, tx):
    g = _gen(T, 18)
    x, w = (T.randn((r, 400), generator=g, device="cuda").to(_type(T, tx)) for r in (300, 270))
    x[131, 390], x[7, 0], w[9, 3] = -float("inf"), float("inf"), float("inf")
    a, sa, b, sb = _empty8(T, 300, 400, "e4m3"), T.empty((4, 300), device="cuda"), _empty8(T, 270, 400, "e4m3"), T.empty((4, 270), device="cuda")
    K.fp8_quantize(x, a, sa)
    K.fp8_quantize(w, b, sb)
    out = T.zeros((300, 270), device="cuda")
    K.fp8_matmul(a, sa, b, sb, out)
    bad = T.zeros((300, 270), dtype=T.bool, device="cuda")
    bad[[7, 131]], bad[:, 9] = True, True
    assert T.isnan(out[bad]).all() and T.isfinite(out[~bad]).all()


# ---- 8-bit product ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("M,N,Kd", [(130, 700, 2050), (3000, 2502, 125), (30_000, 60, 300), (2600, 2048, 2300), (3, 40, 700)])
@pytest.mark.parametrize("ba,bb,fmt", [(1, 1, "e4m3"), (1, 128, "e4m3"), (128, 1, "e5m2"), (128, 128, "e5m2")])
def test_product_of_scales_far_from_one(T, K, M, N, Kd, ba, bb, fmt):
    """Wherever the values' products lie in fp32's range, the scales' own product need not: it may fall below the normal numbers or beyond
    the largest.  Every kind of pair meets in one tile; rows of zeros stay zero under any scale."""
    g = _gen(T, M + N + ba)
    made = []
    for rows, block in ((M, ba), (N, bb)):
        q = _empty8(T, rows, Kd, fmt)
        q.copy_(T.randn((rows, Kd), generator=g, device="cuda").to(q.dtype))
        e = T.tensor([0, -60, 60, -85, 90, -118, 110, 1, -64, 64], device="cuda")[T.randint(0, 10, ((rows + block - 1) // block,), generator=g, device="cuda")]
        s = T.exp2(e.float())[None, :] * (1 + T.rand(((Kd + 127) // 128, e.numel()), generator=g, device="cuda"))
        if rows > 2:
            q.view(T.uint8)[1] = 0
        made += [q, s.contiguous()]
    va, vb = _stands_for(T, *made[:2]), _stands_for(T, *made[2:])
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    out, status = T.full((M, N), 9.0, device="cuda"), T.zeros(1, dtype=T.int32, device="cuda")
    K.fp8_matmul(*made, out, status=status)
    fits = size < 2.0 ** 127
    # (each block's product with a scale and its addition may also be off by half the smallest step, 2^-150)
    tol = _product_tol(T, va, vb, Kd) + 4 * ((Kd + 127) // 128) * 2.0 ** -150
    assert status.item() == 0 and fits.any()
    if M > 128:                                   # (the smallest case may have one pair of scales only)
        assert bool((want[fits].abs() < 2.0 ** -100).any()) and bool((want[fits].abs() > 2.0 ** 60).any())
    _check(T, out[fits], want[fits], tol[fits])
    if M > 2 and N > 2:
        assert (out[1] == 0).all() and (out[:, 1] == 0).all()


def test_product_waits_that_run_out_leave_the_context_usable(T, K):
    """Limits so short that a wait runs out anywhere in any form of the kernel: the call reports KGE_ERR_TIMEOUT (or got by), and the next one is
    right."""
    sizes = [(130, 700, 2050, 1), (3000, 2502, 125, 128), (30_000, 60, 300, 128), (2600, 2048, 2300, 128), (2600, 2048, 2300, 1)]
    ran_out = 0
    for M, N, Kd, bb in sizes:
        g = _gen(T, M)
        a, sa = _empty8(T, M, Kd, "e4m3"), T.empty(((Kd + 127) // 128, M), device="cuda")
        b, sb = _empty8(T, N, Kd, "e4m3"), T.empty(((Kd + 127) // 128, N if bb == 1 else (N + 127) // 128), device="cuda")
        K.fp8_quantize(T.randn((M, Kd), generator=g, device="cuda"), a, sa)
        K.fp8_quantize(T.randn((N, Kd), generator=g, device="cuda"), b, sb, block_rows=bb)
        want, out, status = T.empty((M, N), device="cuda"), T.empty((M, N), device="cuda"), T.zeros(1, dtype=T.int32, device="cuda")
        K.fp8_matmul(a, sa, b, sb, want, status=status)
        assert status.item() == 0
        try:
            for tries in (1, 1, 1, 1, 2, 4, 8, 16, 64):
                assert K.lib().kge_debug_set_product_wait_limit(tries) == 0
                K.fp8_matmul(a, sa, b, sb, out, status=status)
                assert status.item() in (0, -11)
                ran_out += status.item() != 0
                if status.item() == 0:
                    assert T.equal(out, want)
                status.zero_()
        finally:
            K.lib().kge_debug_set_product_wait_limit(0)
        out.fill_(float("nan"))
        K.fp8_matmul(a, sa, b, sb, out, status=status)
        assert status.item() == 0 and T.equal(out, want)
    assert ran_out


# ---- gradient --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,E,kind", [(40, 3, "one"), (300, 5, "one"), (700, 40, "zipf"), (1024, 9, "blocks"), (2048, 8192, "one"), (3000, 7, "zipf"),
                                      (3000, 2, "one"), (20_000, 30, "zipf"), (140_000, 11, "zipf"), (140_000, 3, "one")])
@pytest.mark.parametrize("d", [1, 2, 4, 8, 16, 24, 64, 128, 256, 300, 512, 1024, 2304])
def test_grad_adds_in_an_order_that_follows_the_ids_alone(T, K, n, E, kind, d):
    """The same values in rows apart, rows shifted off their alignment and other types give the same bits, also where an id has a long run."""
    if n * d > 40_000_000:
        n = 40_000_000 // d
    g = _gen(T, n + d)
    ids = _id_list(T, g, kind, n, E)
    values = T.randn((n, d), generator=g, device="cuda").to(T.bfloat16)
    want = T.empty((E, d), device="cuda")
    K.embedding_grad(ids, values, want, scale=0.75)
    for tg, to, extra, shift in ((T.bfloat16, T.float32, 0, 1), (T.bfloat16, T.float32, 0, 2), (T.bfloat16, T.float32, 4, 4), (T.float32, T.float32, 0, 0),
                                 (T.float32, T.float32, 1, 0), (T.float32, T.float32, 0, 2), (T.bfloat16, T.bfloat16, 0, 0), (T.float32, T.float16, 3, 1)):
        grads, out = _strided(T, n, d, tg, extra, shift), _strided(T, E, d, to, extra, shift)
        grads.copy_(values)
        K.embedding_grad(ids, grads, out, scale=0.75)
        assert T.equal(out, want.to(to)), (tg, to, extra, shift, int((out != want.to(to)).any(0).sum()))


@pytest.mark.parametrize("n,E,kind", [(900, 4, "one"), (1024, 50, "zipf"), (2048, 9000, "one"), (3000, 2, "one"), (5000, 600, "blocks"), (60_000, 70_000, "zipf"),
                                      (65_536, 3, "one"), (65_537, 900, "zipf"), (131_071, 40, "one"), (131_072, 40, "one"), (140_003, 5000, "blocks"),
                                      (200_000, 2_100_000, "zipf"), (300_000, 5000, "one"), (450_000, 77, "padded")])
@pytest.mark.parametrize("d,tg,to", [(256, "bf16", "f32"), (32, "f32", "f32"), (36, "bf16", "f32"), (12, "f16", "f32"), (5, "f32", "f32"), (4, "bf16", "bf16")])
def test_grad_of_whole_numbers_is_exact(T, K, n, E, kind, d, tg, to):
    """Sums of small whole numbers stay below 2^24 (450,000 times 8), so every order of fp32 additions gives the same: no row may be lost or
    counted twice, however long its id's run."""
    if E * d > 30_000_000:
        E = 30_000_000 // d
    g = _gen(T, n + d + E)
    ids = _id_list(T, g, kind, n, E)
    grads = T.randint(-6, 9, (n, d), generator=g, device="cuda").to(_type(T, tg))
    out, old = T.full((E, d), float("nan"), device="cuda", dtype=_type(T, to)), T.randint(-50, 50, (E, d), generator=g, device="cuda").to(_type(T, to))
    keep = ids >= 0
    want = T.zeros((E, d), dtype=T.float64, device="cuda").index_add_(0, ids[keep].long(), grads[keep].double())
    assert want.abs().max() < 2 ** 24
    K.embedding_grad(ids, grads, out)
    assert T.equal(out, want.to(out.dtype)), int((out.double() != want).any(1).sum())
    more = old.clone()
    K.embedding_grad(ids, grads, more, accumulate=True)
    assert T.equal(more, (want + old.double()).to(more.dtype))


@pytest.mark.parametrize("n,E,d,kind,tg", [(24_576, 100_000, 128, "zipf", "f32"), (200_000, 500_000, 12, "zipf", "f32"), (300_000, 5000, 36, "one", "bf16"),
                                           (500_000, 2, 16, "one", "bf16"), (150_000, 1000, 256, "zipf", "bf16"), (1000, 3, 40, "one", "f32")])
def test_grad_is_as_near_as_its_depth_of_additions(T, K, n, E, d, kind, tg):
    """A value passes through at most: the rows of two chunks (8 or 32 each) in turn, the chunks that are joined in a CTA, every 16th partial
    sum of its run, and 16 stripes; in a list of one launch, every 51st row of its run (256 threads over five packs) and the 51 sums of those.
    Each addition rounds once."""
    g = _gen(T, n)
    ids = _id_list(T, g, kind, n, E)
    grads = T.randn((n, d), generator=g, device="cuda").to(_type(T, tg))
    out = T.empty((E, d), device="cuda")
    K.embedding_grad(ids, grads, out)
    zeros = lambda: T.zeros((E, d), dtype=T.float64, device="cuda")
    want, size = zeros().index_add_(0, ids.long(), grads.double()), zeros().index_add_(0, ids.long(), grads.double().abs())
    chunk, group = 8 if n < 1 << 17 else 32, 1024 // d if 1024 % d == 0 else 1
    depth = 2 * chunk + group + -(-n // (chunk * group * 16)) + -(-2 * group // 16) + 16 if n > 2048 else -(-n // 51) + 51
    _check(T, out, want, depth * U * size, kind)


def test_grad_of_rows_wider_than_a_grid_is_high(T, K):
    """65,535 times 64 columns and more in a list whose ids are joined from partial sums."""
    n, d = 1025, 65_535 * 64 + 72
    ids = T.ones(n, dtype=T.int32, device="cuda")
    ids[::100] = 0
    grads = T.empty((n, d), dtype=T.bfloat16, device="cuda")
    for i in range(n):
        grads[i] = T.arange(d, device="cuda") % 7 + i % 3
    out = T.full((3, d), float("nan"), device="cuda")
    K.embedding_grad(ids, grads, out)
    at = T.arange(n, device="cuda")
    base = (T.arange(d, device="cuda") % 7).float()
    for e in range(2):
        mine = at[ids == e]
        assert T.equal(out[e], base * len(mine) + float((mine % 3).sum()))
    assert (out[2] == 0).all()


# ---- arrays beyond 2^31 elements -------------------------------------------------------------------------------------

def _halves_of(groups, seed, step, site):
    """The documented 16-bit numbers of these groups of eight elements."""
    x = [np.asarray(groups, dtype=np.uint64)] + [np.full(len(groups), v, dtype=np.uint64) for v in (step & 0xFFFFFFFF, step >> 32, (1 << 31) + site)]
    k0, k1, low, m = seed & 0xFFFFFFFF, seed >> 32, np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> m) ^ x[1] ^ np.uint64(k0), q & low, (p >> m) ^ x[3] ^ np.uint64(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack([h for w in x for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 1).reshape(-1)


def test_dropout_of_2_to_the_34_elements(T, K):
    n = 1 << 34
    x = T.ones(n, dtype=T.bfloat16, device="cuda")
    K.dropout(x, x, 0.25, 77, 5, site=3)
    for at in (0, (1 << 31) - 4096, (1 << 32) - 4096, (1 << 33) - 4096, n - 8192):
        keep = T.from_numpy(_halves_of(np.arange(at // 8, at // 8 + 1024), 77, 5, 3) >= 16384).cuda()
        assert T.equal(x[at:at + 8192], T.where(keep, 4.0 / 3.0, 0.0).to(T.bfloat16))
    del x


def test_quantize_and_product_beyond_two_to_the_31_elements(T, K):
    """2.2 M rows of 1,024: values in and out in both orientations, then as an operand; and an output of 70,000 x 32,000."""
    g = _gen(T, 31)
    rows, cols = 2_200_000, 1024
    x = T.empty((rows, cols), dtype=T.bfloat16, device="cuda")
    for r in range(0, rows, 100_000):
        x[r:r + 100_000] = T.randn((100_000, cols), generator=g, device="cuda")
    q, s = _empty8(T, rows, cols, "e4m3"), T.empty((8, rows), device="cuda")
    qt, st = _empty8(T, cols, rows, "e4m3"), T.empty(((rows + 127) // 128, cols), device="cuda")
    K.fp8_quantize(x, q, s, qt, st)
    for r in (0, 2_097_152 - 128, 2_097_152, rows // 128 * 128 - 128):         # (2,097,152 rows are 2^31 values)
        some = x[r:r + 256]
        want, ws = _quantized(T, some, "e4m3", 1, False)
        assert T.equal(q[r:r + 256].float().double(), want) and T.equal(s[:, r:r + 256], ws)
        want, ws = _quantized(T, some.t(), "e4m3", 1, False)
        assert T.equal(qt[:, r:r + 256].float().double(), want) and T.equal(st[r // 128:r // 128 + 2], ws)
    del x, qt, st
    w, ws = _empty8(T, 40, cols, "e4m3"), T.empty((8, 1), device="cuda")
    K.fp8_quantize(T.randn((40, cols), generator=g, device="cuda"), w, ws, block_rows=128)
    out, status = T.empty((rows, 40), device="cuda"), T.zeros(1, dtype=T.int32, device="cuda")
    K.fp8_matmul(q, s, w, ws, out, status=status)
    vw = _stands_for(T, w, ws)
    for r in (0, 2_097_152 - 150, rows - 300):
        va = _stands_for(T, q[r:r + 300], s[:, r:r + 300])
        _check(T, out[r:r + 300], va @ vw.t(), _product_tol(T, va, vw, cols))
    del out, w
    a, sa, b, sb = q[:70_000, :64], s[:1, :70_000].contiguous(), q[100_000:132_000, :64], s[:1, 100_000:132_000].contiguous()
    out = T.empty((70_000, 32_000), dtype=T.bfloat16, device="cuda")
    K.fp8_matmul(a, sa, b, sb, out, status=status)
    vb = _stands_for(T, b, sb)
    for r in (0, 67_100, 69_800):                                              # (67,109 rows are 2^31 values)
        va = _stands_for(T, a[r:r + 200], sa[:, r:r + 200])
        _check(T, out[r:r + 200], va @ vb.t(), _product_tol(T, va, vb, 64))
    assert status.item() == 0


def test_lookup_and_grad_of_more_than_two_to_the_31_elements_in_a_list(T, K):
    n, E, d = 8_500_000, 1000, 256
    g = _gen(T, 32)
    ids = T.randint(0, E, (n,), generator=g, device="cuda", dtype=T.int32)
    table = T.randint(-9, 10, (E, d), generator=g, device="cuda").to(T.bfloat16)
    rows = T.empty((n, d), dtype=T.bfloat16, device="cuda")
    K.embedding_lookup(table, ids, rows, scale=2.0)
    out, want = T.empty((E, d), device="cuda"), T.zeros((E, d), dtype=T.float64, device="cuda")
    for r in range(0, n, 500_000):
        some = rows[r:r + 500_000]
        assert T.equal(some, table[ids[r:r + 500_000].long()] * 2)
        want.index_add_(0, ids[r:r + 500_000].long(), some.double())
    K.embedding_grad(ids, rows, out)
    assert T.equal(out.double(), want)                    # (whole numbers: 8,500 rows of at most 18 to an id or so)
