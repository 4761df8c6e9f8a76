"""Refusals of the operators for a residual block, without a GPU: every bad argument is turned down on the host before anything is launched
(the pointers below are never followed), and the binding turns down tensors that do not fit."""
import ctypes as C

import pytest

from test_row_operators_cpu import BF16, E4M3, F16, F32, K, PTR  # noqa: F401

QUANT = dict(x=PTR, x_type=F32, rows=4, cols=64, ldx=64, q=PTR, ldq=64, scales=PTR, stream=None)
MATMUL = dict(a=PTR, lda=64, a_scales=PTR, b=PTR, ldb=64, b_scales=PTR, addend=None, ld_addend=0, out=PTR, out_type=F32, ld_out=32, M=16, N=32, K=64,
              status=None, stream=None)
BLOCK = dict(x=PTR, y=PTR, gate=PTR, post_weight=PTR, post_bias=PTR, scale=PTR, pre_weight=PTR, pre_bias=PTR, ldx=8, ldy=8, ld_gate=8, x_type=F32, block_type=BF16,
             gate_act=1, layer=1)
NORM = dict(n=4, d=8, h=PTR, ldh=8, z=PTR, z_int8=0, ldz=8, z_scales=None, eps=1e-6, stats=PTR, stream=None)
GRADS = dict(dx=PTR, dy=PTR, dgate=PTR, dpost_weight=PTR, dpost_bias=PTR, dscale=PTR, dpre_weight=PTR, dpre_bias=PTR, ld_dx=8, ld_dy=8, ld_dgate=8)
GRAD = dict(n=4, d=8, stats=PTR, dz=PTR, ld_dz=8, dh=PTR, ld_dh=8, accumulate=0, scratch=PTR, scratch_bytes=1 << 30, stream=None)
TENSOR = dict(param=PTR, grad=PTR, m=PTR, v=PTR, m_scales=PTR, v_scales=PTR, copy=None, n=10, param_type=F32, grad_type=F32, copy_type=0, weight_decay=0.0)
STEP = dict(bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=0, step_dev=None, lr_dev=None, grad_scale_dev=None, seed=1, stream=None)


def _plain(K, name, base, over):
    return getattr(K.lib(), name)(*dict(base, **over).values())


@pytest.mark.parametrize("over", [dict(x=None), dict(q=None), dict(scales=None), dict(x_type=E4M3), dict(rows=-1), dict(cols=-1), dict(ldx=63), dict(ldq=48), dict(ldq=72),
                                  dict(q=PTR + 8), dict(scales=PTR + 2), dict(x=PTR + 2), dict(rows=1 << 31), dict(cols=1 << 31, ldx=1 << 31, ldq=1 << 31)])
def test_int8_quantize_refuses(K, over):
    assert _plain(K, "kge_int8_quantize", QUANT, over) == -1


@pytest.mark.parametrize("over,code", [(dict(a=None), -1), (dict(b=None), -1), (dict(a_scales=None), -1), (dict(b_scales=None), -1), (dict(out=None), -1), (dict(out_type=E4M3), -1),
                                       (dict(M=-1), -1), (dict(N=-1), -1), (dict(K=0), -1), (dict(K=65), -1), (dict(lda=72), -1), (dict(ldb=48), -1), (dict(ld_out=31), -1),
                                       (dict(a=PTR + 8), -1), (dict(b=PTR + 4), -1), (dict(out=PTR + 2), -1), (dict(addend=PTR, ld_addend=31), -1), (dict(status=PTR + 2), -1),
                                       (dict(addend=PTR + 2, ld_addend=32), -1), (dict(M=1 << 31), -1), (dict(a_scales=PTR + 1), -1),
                                       (dict(K=131_072, lda=131_072, ldb=131_072), -5)])
def test_int8_matmul_refuses(K, over, code):
    assert _plain(K, "kge_int8_matmul", MATMUL, over) == code


def _norm(K, block=(), **over):
    from paper_2211_12281_b200.binding import KGE_NORM_BLOCK
    return K.lib().kge_block_norm(KGE_NORM_BLOCK.pack(*[v or 0 for v in dict(BLOCK, **dict(block)).values()]), *dict(NORM, **over).values())


@pytest.mark.parametrize("block,over", [
    (dict(x=None), {}), (dict(x_type=E4M3), {}), (dict(block_type=7), {}), (dict(layer=2), {}), (dict(gate_act=3), {}), (dict(gate_act=-1), {}), (dict(ldx=7), {}), (dict(ldy=7), {}),
    (dict(ld_gate=7), {}), (dict(x=PTR + 2), {}), (dict(y=PTR + 1), {}), (dict(gate=PTR + 1), {}), (dict(y=None), {}), (dict(post_weight=None), {}), (dict(pre_weight=None), {}),
    (dict(scale=PTR + 2), {}), ({}, dict(n=-1)), ({}, dict(n=1 << 31)), ({}, dict(d=0)), ({}, dict(d=(1 << 31) - 1)), ({}, dict(h=None, z=None)), ({}, dict(ldh=7)), ({}, dict(ldz=7)),
    ({}, dict(h=PTR + 2)), ({}, dict(z=PTR + 1)), ({}, dict(z_int8=1)), ({}, dict(z_int8=2)), ({}, dict(z_int8=1, z_scales=PTR + 2)), ({}, dict(eps=-1.0)), ({}, dict(eps=float("nan"))),
    ({}, dict(eps=float("inf"))), ({}, dict(stats=PTR + 4))])
def test_block_norm_refuses(K, block, over):
    assert _norm(K, block, **over) == -1


def _grad(K, block=(), grads=(), **over):
    from paper_2211_12281_b200.binding import KGE_NORM_BLOCK, KGE_NORM_GRADS
    a = dict(GRAD, **over)
    return K.lib().kge_block_norm_grad(KGE_NORM_BLOCK.pack(*[v or 0 for v in dict(BLOCK, **dict(block)).values()]), a["n"], a["d"], a["stats"], a["dz"], a["ld_dz"], a["dh"], a["ld_dh"],
                                       KGE_NORM_GRADS.pack(*[v or 0 for v in dict(GRADS, **dict(grads)).values()]), a["accumulate"], a["scratch"], a["scratch_bytes"], a["stream"])


@pytest.mark.parametrize("block,grads,over,code", [
    (dict(x=None), {}, {}, -1), (dict(x_type=5), {}, {}, -1), (dict(block_type=E4M3), {}, {}, -1), (dict(layer=-1), {}, {}, -1), (dict(gate_act=3), {}, {}, -1), (dict(ldx=7), {}, {}, -1),
    (dict(y=None), {}, {}, -1), (dict(gate=None), {}, {}, -1), (dict(post_weight=None), {}, {}, -1), (dict(scale=None), {}, {}, -1), (dict(pre_weight=None), {}, {}, -1), ({}, dict(ld_dx=7), {}, -1),
    ({}, dict(ld_dy=7), {}, -1), ({}, dict(ld_dgate=7), {}, -1), ({}, dict(dx=PTR + 2), {}, -1), ({}, dict(dy=PTR + 1), {}, -1), ({}, dict(dscale=PTR + 1), {}, -1),
    ({}, {}, dict(n=-1), -1), ({}, {}, dict(d=0), -1), ({}, {}, dict(stats=None), -1), ({}, {}, dict(stats=PTR + 8), -1), ({}, {}, dict(dz=None, dh=None), -1), ({}, {}, dict(dz=None), -1),
    ({}, {}, dict(dz=PTR + 1), -1), ({}, {}, dict(dh=PTR + 2), -1), ({}, {}, dict(ld_dz=7), -1), ({}, {}, dict(ld_dh=7), -1), ({}, {}, dict(accumulate=2), -1),
    ({}, {}, dict(scratch=None), -4), ({}, {}, dict(scratch=PTR + 128), -4), ({}, {}, dict(scratch_bytes=127), -4)])
def test_block_norm_grad_refuses(K, block, grads, over, code):
    assert _grad(K, block, grads, **over) == code


def _adamw(K, tensor=(), count=1, **over):
    from paper_2211_12281_b200.binding import KgeAdamwTensor
    a = dict(STEP, **over)
    at = (KgeAdamwTensor * 1)(KgeAdamwTensor(**dict(TENSOR, **dict(tensor))))
    return K.lib().kge_adamw(at, count, *a.values())


@pytest.mark.parametrize("tensor,over,code", [
    (dict(param=None), {}, -1), (dict(m=None), {}, -1), (dict(v=None), {}, -1), (dict(n=-1), {}, -1), (dict(param_type=E4M3), {}, -1), (dict(grad_type=5), {}, -1), (dict(param=PTR + 2), {}, -1),
    (dict(grad=PTR + 1), {}, -1), (dict(m=PTR + 2), {}, -1), (dict(copy=PTR, copy_type=F32), {}, -1), (dict(copy=PTR + 1, copy_type=F16), {}, -1), (dict(weight_decay=float("nan")), {}, -1),
    (dict(n=(1 << 40) + 1), {}, -5), (dict(m_scales=None), dict(bits=8), -1), (dict(v_scales=PTR + 2), dict(bits=8), -1), ({}, dict(bits=16), -1), ({}, dict(lr=float("inf")), -1),
    ({}, dict(beta1=1.0), -1), ({}, dict(beta2=-0.1), -1), ({}, dict(beta2=float("nan")), -1), ({}, dict(eps=0.0), -1), ({}, dict(eps=1e-50), -1), ({}, dict(eps=float("inf")), -1),
    ({}, dict(grad_scale=float("nan")), -1), ({}, dict(step=1 << 62), -1), ({}, dict(step_dev=PTR + 4), -1), ({}, dict(lr_dev=PTR + 2), -1), ({}, dict(grad_scale_dev=PTR + 1), -1),
    ({}, dict(count=-1), -1)])
def test_adamw_refuses(K, tensor, over, code):
    count = over.pop("count", 1) if "count" in over else 1
    assert _adamw(K, tensor, count, **over) == code


def test_calls_on_nothing_return_at_once(K):
    assert _plain(K, "kge_int8_quantize", QUANT, dict(rows=0, x=None)) == 0
    assert _plain(K, "kge_int8_matmul", MATMUL, dict(M=0, a=None)) == 0
    assert _norm(K, dict(x=None), n=0) == 0
    assert _grad(K, n=0, accumulate=1, stats=None, scratch=None) == 0
    assert _adamw(K, count=0) == 0
    assert _adamw(K, dict(grad=None, param=None)) == 0 and _adamw(K, dict(n=0, param=None)) == 0


def test_mirrors_have_the_header_layout(K, tmp_path):
    """Sizes and places of the structures' fields as a C compiler lays them out."""
    import subprocess
    from pathlib import Path
    from paper_2211_12281_b200.binding import KGE_NORM_BLOCK, KGE_NORM_GRADS, KgeAdamwTensor
    src = tmp_path / "layout.c"
    src.write_text("""#include <stddef.h>
#include <stdio.h>
#include "kge.h"
int main(void) {
    printf("%zu %zu %zu ", sizeof(kge_adamw_tensor), offsetof(kge_adamw_tensor, n), offsetof(kge_adamw_tensor, weight_decay));
    printf("%zu %zu %zu %zu ", sizeof(kge_norm_block), offsetof(kge_norm_block, pre_bias), offsetof(kge_norm_block, ldx), offsetof(kge_norm_block, layer));
    printf("%zu %zu %zu\\n", sizeof(kge_norm_grads), offsetof(kge_norm_grads, dpre_bias), offsetof(kge_norm_grads, ld_dgate));
    return 0;
}
""")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", str(Path(__file__).resolve().parent.parent / "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got[:3] == [C.sizeof(KgeAdamwTensor), KgeAdamwTensor.n.offset, KgeAdamwTensor.weight_decay.offset]
    assert got[3:] == [KGE_NORM_BLOCK.size, 56, 64, 100, KGE_NORM_GRADS.size, 56, 80]


def test_scratch_of_gradients_holds_every_share(K):
    for n, d in ((1, 1), (5, 300), (100_000, 256), (100_000, 4096), (3, 20_000)):
        assert K.block_norm_grad_scratch_bytes(n, d) >= 4 * 4 * d
    assert K.block_norm_grad_scratch_bytes(0, 8) == 0 and K.block_norm_grad_scratch_bytes(8, 0) == 0
    with pytest.raises(K.KgeError):
        K.block_norm_grad_scratch_bytes(1 << 33, 8)


def test_binding_refuses_tensors_that_do_not_fit(K):
    import torch
    f, i8 = (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.int8))
    x, w = f(4, 8), f(8)
    e4, e5 = torch.zeros(300, dtype=torch.float8_e4m3fn), torch.zeros(300, dtype=torch.float8_e5m2)
    bad = [lambda: K.int8_quantize(x, i8(4, 8), f(4)),                                            # not on a GPU
           lambda: K.int8_quantize(x, i8(4, 9), f(4)), lambda: K.int8_quantize(x, i8(4, 8), f(3)), lambda: K.int8_quantize(x, f(4, 8), f(4)),
           lambda: K.int8_quantize(x.double(), i8(4, 8), f(4)),
           lambda: K.int8_matmul(i8(4, 16), f(4), i8(8, 32), f(8), f(4, 8)), lambda: K.int8_matmul(i8(4, 16), f(4), i8(8, 16), f(7), f(4, 8)),
           lambda: K.int8_matmul(i8(4, 16), f(4), i8(8, 16), f(8), f(4, 8), addend=f(4, 8).half()), lambda: K.int8_matmul(i8(4, 16), f(4, 1), i8(8, 16), f(8), f(4, 8)),
           lambda: K.block_norm(x, z=f(4, 8), pre_weight=w),                                      # not on a GPU
           lambda: K.block_norm(x, z=f(4, 7), pre_weight=w), lambda: K.block_norm(x, z=f(4, 8), pre_weight=f(7)), lambda: K.block_norm(x, z=f(4, 8), pre_weight=w.half()),
           lambda: K.block_norm(x, z=f(4, 8), pre_weight=w, y=f(4, 8).half()), lambda: K.block_norm(x, z=f(4, 8), pre_weight=w, y=x, h=f(4, 8).half()),
           lambda: K.block_norm(x, z=f(4, 8), pre_weight=w, y=x, gate=f(4, 1)), lambda: K.block_norm(x, z=f(4, 8), pre_weight=w, y=x, gate=x, gate_act="tanh"),
           lambda: K.block_norm(x, z=f(4, 8), pre_weight=w, kind="batch"), lambda: K.block_norm(x, z=i8(4, 8), pre_weight=w), lambda: K.block_norm(x, z=f(4, 8), pre_weight=w, z_scales=f(4)),
           lambda: K.block_norm(x, z=f(4, 8), pre_weight=w, stats=f(4, 2)), lambda: K.block_norm(x.t(), z=f(8, 4), pre_weight=f(4)),
           lambda: K.block_norm_grad(x, f(4, 4), f(4, 8), dz=f(4, 8), pre_weight=w), lambda: K.block_norm_grad(x, None, f(4, 8), dz=f(4, 8), pre_weight=w),
           lambda: K.block_norm_grad(x, f(4, 4), f(4, 8), dz=f(3, 8), pre_weight=w), lambda: K.block_norm_grad(x, f(4, 4), f(4, 8).half(), dz=f(4, 8), pre_weight=w),
           lambda: K.block_norm_grad(x, f(4, 4), f(4, 8), dz=f(4, 8), pre_weight=w, dpre_weight=f(9)),
           lambda: K.AdamW([f(8)], [f(8)], [f(8)], [f(8)]),                                       # not on a GPU
           lambda: K.AdamW([f(8)], [f(8)], [f(8)], []), lambda: K.AdamW([f(8)], [f(8)], [f(7)], [f(8)]), lambda: K.AdamW([f(8)], [f(8)], [f(8)], [f(8).half()]),
           lambda: K.AdamW([f(300)], [f(300)], [e4], [e5]), lambda: K.AdamW([f(300)], [f(300)], [e4], [e5], [f(2)], [f(3)]),
           lambda: K.AdamW([f(300)], [f(300)], [e4], [e4], [f(3)], [f(3)]), lambda: K.AdamW([f(8)], [f(8)], [f(8)], [f(8)], copies=[f(8)]),
           lambda: K.AdamW([f(8)], [f(8)], [f(8)], [f(8)], weight_decay=[0.1, 0.1]), lambda: K.AdamW([f(8).double()], [f(8)], [f(8)], [f(8)])]
    for k, call in enumerate(bad):
        with pytest.raises(K.KgeError) as e:
            call()
        assert e.value.code == -1, k
