"""Refusals of the operators on rows, without a GPU: every bad argument is turned down on the host before anything is launched
(the pointers below are never followed), and the binding turns down tensors that do not fit."""
import pytest

PTR = 1 << 20          # an aligned address that nothing reads
F32, BF16, F16, E4M3, E5M2 = range(5)


@pytest.fixture(scope="module")
def K():
    from paper_2211_12281_b200 import build
    build.build()
    import paper_2211_12281_b200 as K
    return K


def _call(K, name, order, base, /, **over):
    args = dict(base, **over)
    return getattr(K.lib(), name)(*[args[k] for k in order])


LOOKUP = dict(table=PTR, table_type=F32, rows=10, dim=8, ld_table=8, ids=PTR, n=4, scale=1.0, padding_id=-1, out=PTR, out_type=F32, ld_out=8,
              status=None, stream=None)
GRAD = dict(ids=PTR, n=4000, grads=PTR, grads_type=F32, ld_grads=8, scale=1.0, padding_id=-1, accumulate=0, table_grad=PTR, table_type=F32, rows=10,
            dim=8, ld_table=8, scratch=PTR, scratch_bytes=1 << 30, status=None, stream=None)
DROPOUT = dict(x=PTR, x_type=F32, residual=None, out=PTR, out_type=F32, n=8, p=0.1, seed=1, step=0, step_dev=None, site=0, stream=None)
QUANT = dict(x=PTR, x_type=F32, rows=4, cols=64, ldx=64, fp8_type=E4M3, block_rows=1, pow2=0, q=PTR, ldq=64, scales=PTR, qt=None, ldqt=0,
             scales_t=None, stream=None)
MATMUL = dict(a=PTR, a_type=E4M3, lda=64, a_scales=PTR, a_block=1, b=PTR, b_type=E4M3, ldb=64, b_scales=PTR, b_block=128, addend=None, ld_addend=0,
              out=PTR, out_type=F32, ld_out=32, M=16, N=32, K=64, status=None, stream=None)


@pytest.mark.parametrize("over", [dict(table=None), dict(ids=None), dict(out=None), dict(table_type=E4M3), dict(out_type=7), dict(rows=0),
                                  dict(rows=1 << 31), dict(dim=0), dict(ld_table=7), dict(ld_out=7), dict(n=-1), dict(table=PTR + 2),
                                  dict(ids=PTR + 1), dict(out=PTR + 1), dict(status=PTR + 2)])
def test_lookup_refuses(K, over):
    assert _call(K, "kge_embedding_lookup", LOOKUP, LOOKUP, **over) == -1


@pytest.mark.parametrize("over,code", [(dict(ids=None), -1), (dict(grads=None), -1), (dict(table_grad=None), -1), (dict(grads_type=E5M2), -1),
                                       (dict(table_type=-1), -1), (dict(rows=0), -1), (dict(dim=0), -1), (dict(ld_grads=7), -1),
                                       (dict(ld_table=7), -1), (dict(n=-1), -1), (dict(accumulate=2), -1), (dict(grads=PTR + 2), -1),
                                       (dict(table_grad=PTR + 1), -1), (dict(scratch=None), -4), (dict(scratch=PTR + 128), -4),
                                       (dict(scratch_bytes=16), -4)])
def test_grad_refuses(K, over, code):
    assert _call(K, "kge_embedding_grad", GRAD, GRAD, **over) == code


@pytest.mark.parametrize("over", [dict(x=None), dict(out=None), dict(x_type=E4M3), dict(out_type=9), dict(n=-1), dict(n=(1 << 34) + 1), dict(p=-0.1),
                                  dict(p=1.5), dict(p=float("nan")), dict(site=-1), dict(x=PTR + 2), dict(residual=PTR + 1), dict(step_dev=PTR + 4)])
def test_dropout_refuses(K, over):
    assert _call(K, "kge_dropout", DROPOUT, DROPOUT, **over) == -1


@pytest.mark.parametrize("over", [dict(x=None), dict(q=None), dict(scales=None), dict(x_type=E4M3), dict(fp8_type=F32), dict(block_rows=64),
                                  dict(pow2=2), dict(ldx=63), dict(ldq=48), dict(ldq=72), dict(q=PTR + 8), dict(rows=-1), dict(cols=-1),
                                  dict(qt=PTR, ldqt=16, scales_t=None), dict(qt=PTR, ldqt=8, scales_t=PTR), dict(qt=PTR + 4, ldqt=16, scales_t=PTR)])
def test_quantize_refuses(K, over):
    assert _call(K, "kge_fp8_quantize", QUANT, QUANT, **over) == -1


@pytest.mark.parametrize("over", [dict(a=None), dict(b=None), dict(a_scales=None), dict(b_scales=None), dict(out=None), dict(a_type=BF16), dict(b_type=F32),
                                  dict(out_type=E4M3), dict(a_block=2), dict(b_block=64), dict(M=-1), dict(N=-1), dict(K=0), dict(K=65), dict(lda=72),
                                  dict(ldb=48), dict(ld_out=31), dict(a=PTR + 8), dict(b=PTR + 4), dict(out=PTR + 2), dict(addend=PTR, ld_addend=31),
                                  dict(addend=PTR + 2, ld_addend=32), dict(M=1 << 31)])
def test_matmul_refuses(K, over):
    assert _call(K, "kge_fp8_matmul", MATMUL, MATMUL, **over) == -1


def test_calls_on_nothing_return_at_once(K):
    assert _call(K, "kge_embedding_lookup", LOOKUP, LOOKUP, n=0, ids=None, out=None, table=None) == 0
    assert _call(K, "kge_embedding_grad", GRAD, GRAD, n=0, ids=None, grads=None, accumulate=1, scratch=None) == 0
    assert _call(K, "kge_dropout", DROPOUT, DROPOUT, n=0, x=None, out=None) == 0
    assert _call(K, "kge_fp8_quantize", QUANT, QUANT, rows=0) == 0
    assert _call(K, "kge_fp8_matmul", MATMUL, MATMUL, M=0, a=None) == 0


def test_binding_features_in_8_bits_refuses(K):
    h = K.Kge(K.KgeConfig.make(num_entities=100, num_relations=3, dim=32, score="transe", batch=4, num_neg=4, feat_dim=64))
    fn = K.lib().kge_bind_features_fp8
    assert fn(None, PTR, E4M3, 64, PTR, PTR, PTR * 2, None, None, None) == -1
    assert fn(h._h, PTR, E4M3, 64, PTR, PTR, PTR * 2, None, None, None) == -6          # tables not bound
    for feat, code, ld, scales in ((PTR, F32, 64, PTR), (PTR, E4M3, 48, PTR), (PTR, E4M3, 72, PTR), (PTR, E4M3, 64, None), (PTR, E4M3, 64, PTR + 2),
                                   (None, E4M3, 64, PTR)):
        assert fn(h._h, feat, code, ld, scales, PTR, PTR * 2, None, None, None) == -1


def test_binding_features_in_8_bits_takes_gpu_tensors_only(K):
    import torch
    h = K.Kge(K.KgeConfig.make(num_entities=100, num_relations=3, dim=32, score="transe", batch=4, num_neg=4, feat_dim=64))
    with pytest.raises(K.KgeError) as e:
        h.bind_features_fp8(torch.zeros((100, 64), dtype=torch.float8_e4m3fn), torch.zeros((1, 100)), torch.zeros((32, 64)), torch.zeros((32, 64)))
    assert e.value.code == -1 and "GPU" in str(e.value)


def test_scratch_sizes_cover_their_lists(K):
    # a list of (id, position) pairs and partial rows for chunks of ids; short lists keep nothing
    for rows, dim, n in ((10, 8, 1025), (1_000_000, 8, 2049), (91_000_000, 128, 24_576), (100, 256, 600_000)):
        got = K.embedding_grad_scratch_bytes(rows, dim, n)
        assert got >= 8 * n and got % 256 == 0
    assert K.embedding_grad_scratch_bytes(10, 8, 1) == 0 and K.embedding_grad_scratch_bytes(1000, 32, 1024) == 0
    assert K.embedding_grad_scratch_bytes(8192, 32, 2048) == 0 < K.embedding_grad_scratch_bytes(8191, 32, 2048)
    assert K.embedding_grad_scratch_bytes(0, 8, 4) == 0 and K.embedding_grad_scratch_bytes(10, 8, 0) == 0


def test_binding_refuses_tensors_that_do_not_fit(K):
    import torch
    f, i = (lambda *s: torch.zeros(s)), (lambda n: torch.zeros(n, dtype=torch.int32))
    e8 = lambda *s: torch.zeros(s, dtype=torch.float8_e4m3fn)
    bad = [lambda: K.embedding_lookup(f(10, 8), i(4), f(4, 8)),                                   # not on a GPU
           lambda: K.embedding_lookup(f(10, 8), i(4), f(4, 7)),
           lambda: K.embedding_lookup(f(10, 8), i(4).long(), f(4, 8)),
           lambda: K.embedding_lookup(f(10, 8).t(), i(4), f(4, 10)),
           lambda: K.embedding_lookup(f(10, 8).double(), i(4), f(4, 8)),
           lambda: K.embedding_lookup(f(10, 8), i(4), f(4, 8), padding_id=1 << 32),
           lambda: K.embedding_grad(i(4), f(3, 8), f(10, 8)),
           lambda: K.embedding_grad(i(4), f(4, 8), f(10, 9)),
           lambda: K.dropout(f(8), f(9), 0.1, 1),
           lambda: K.dropout(f(8, 8).t(), f(8, 8), 0.1, 1),
           lambda: K.dropout(f(8), f(8), 0.1, 1, residual=f(8).half()),
           lambda: K.dropout(f(8), f(8), 0.1, -1),
           lambda: K.dropout(f(8), f(8), 0.1, 1, step_dev=torch.zeros(0, dtype=torch.int64)),
           lambda: K.fp8_quantize(f(4, 64)),
           lambda: K.fp8_quantize(f(4, 64), e8(4, 64), f(1, 3)),
           lambda: K.fp8_quantize(f(4, 64), e8(4, 64), f(1, 4), block_rows=128),
           lambda: K.fp8_quantize(f(4, 64), f(4, 64), f(1, 4)),
           lambda: K.fp8_matmul(e8(4, 64), f(1, 4), e8(8, 32), f(1, 8), f(4, 8)),
           lambda: K.fp8_matmul(e8(4, 64), f(2, 4), e8(8, 64), f(1, 8), f(4, 8)),
           lambda: K.fp8_matmul(e8(4, 64), f(1, 4), e8(8, 64), f(1, 8), f(4, 8), addend=f(4, 8).half())]
    for call in bad:
        with pytest.raises(K.KgeError) as e:
            call()
        assert e.value.code == -1
