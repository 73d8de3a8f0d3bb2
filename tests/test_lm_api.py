"""The entry points at a language model's ends: exported, and refusing what they should
on the host (no GPU work is issued)."""
import ctypes
import os
import re

import pytest
import torch

from helpers import ROOT, ensure_built


@pytest.fixture(scope="module")
def oz():
    ensure_built()
    import paper_2606_06510_gb300 as oz
    oz.lib()
    return oz


def test_header_and_binding_agree(oz):
    txt = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "oz2_lm.h")).read(), flags=re.S)
    names = set(re.findall(r"^int (oz2_\w+)\(", txt, flags=re.M))
    assert names == set(oz.lm.SIGS)
    raw = ctypes.CDLL(oz.LIB_PATH)
    assert all(hasattr(raw, n) for n in names)
    for n in names:  # as many arguments as the header has
        args = re.search(rf"^int {n}\((.*?)\);", txt, flags=re.M | re.S).group(1).split(",")
        assert len(args) == len(oz.lm.SIGS[n][1]), n
        assert hasattr(oz, n)


BF16, F16, E4M3, F32 = 1, 2, 3, 0
N = None
BIG = (1 << 31) - 256
NAN, INF = float("nan"), float("inf")


def embedding(oz, m=4, n=8, k=8, type=BF16, ids=16, bits=64, E=16, lde=8, scale=1.0, Y=16, ldy=8):
    return oz.lib().oz2_embedding(m, n, k, type, ids, bits, E, lde, scale, Y, ldy, N)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(n=-1), dict(k=-1), dict(type=E4M3), dict(type=9), dict(bits=16), dict(lde=7), dict(ldy=7),
    dict(ids=N), dict(E=N), dict(Y=N), dict(ids=20), dict(bits=32, ids=18), dict(E=17), dict(Y=17), dict(type=F32, Y=18)])
def test_embedding_refuses(oz, bad):
    assert embedding(oz, **bad) == -1


def test_embedding_limits_and_empty(oz):
    assert embedding(oz, m=BIG) == embedding(oz, n=BIG) == embedding(oz, k=BIG, lde=BIG, ldy=BIG) == -6
    assert embedding(oz, m=0, ids=N, Y=N) == embedding(oz, k=0, E=N, Y=N) == 0


def embedding_grad(oz, m=4, n=8, k=8, type=BF16, dY=16, lddy=8, ids=16, bits=64, scale=1.0, dE=16, ldde=8, et=BF16, flags=0):
    return oz.lib().oz2_embedding_grad(m, n, k, type, dY, lddy, ids, bits, scale, dE, ldde, et, flags, N)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(n=-1), dict(k=-1), dict(type=E4M3), dict(bits=8), dict(lddy=7), dict(ldde=7), dict(et=F16),
    dict(et=E4M3), dict(flags=2), dict(dY=N), dict(ids=N), dict(dE=N), dict(dY=17), dict(ids=20), dict(dE=17),
    dict(et=F32, dE=18), dict(type=F32, et=BF16)])
def test_embedding_grad_refuses(oz, bad):
    assert embedding_grad(oz, **bad) == -1


def test_embedding_grad_limits_and_empty(oz):
    assert embedding_grad(oz, m=BIG) == embedding_grad(oz, n=BIG) == -6
    assert embedding_grad(oz, n=0, dE=N) == embedding_grad(oz, k=0, dE=N) == 0
    assert embedding_grad(oz, m=0, dY=N, ids=N, dE=N, flags=1) == 0


def norm(oz, m=4, k=8, type=BF16, X=16, ldx=8, w=16, b=16, wt=BF16, eps=1e-5, center=1, Y=16, ldy=8, mean=N, rstd=N):
    return oz.lib().oz2_layer_norm(m, k, type, X, ldx, w, b, wt, eps, center, Y, ldy, mean, rstd, N)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(k=-1), dict(type=E4M3), dict(wt=F16), dict(wt=E4M3), dict(eps=-1.0), dict(eps=NAN), dict(ldx=7),
    dict(ldy=7), dict(X=N), dict(Y=N), dict(X=17), dict(Y=17), dict(w=17), dict(b=17), dict(wt=F32, w=18), dict(mean=18),
    dict(rstd=18), dict(ldy=9)])
def test_norm_refuses(oz, bad):
    assert norm(oz, **bad) == -1


def test_norm_limits_and_empty(oz):
    assert norm(oz, m=BIG) == norm(oz, k=BIG, ldx=BIG, ldy=BIG) == -6
    assert norm(oz, m=0, X=N, Y=N) == norm(oz, k=0, X=N, Y=N) == 0


def norm_grad(oz, m=4, k=8, type=BF16, dY=16, lddy=8, X=16, ldx=8, mean=16, rstd=16, w=16, wt=BF16, R=16, ldr=8, dX=16,
              lddx=8, dw=16, db=16, flags=0):
    return oz.lib().oz2_layer_norm_grad(m, k, type, dY, lddy, X, ldx, mean, rstd, w, wt, R, ldr, dX, lddx, dw, db, flags, N)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(k=-1), dict(type=E4M3), dict(wt=F16), dict(flags=2), dict(lddy=7), dict(ldx=7), dict(ldr=7),
    dict(lddx=7), dict(dY=N), dict(X=N), dict(rstd=N), dict(dY=17), dict(X=17), dict(R=17), dict(dX=17), dict(dw=18),
    dict(db=18), dict(mean=18), dict(rstd=18), dict(w=17), dict(lddx=9)])
def test_norm_grad_refuses(oz, bad):
    assert norm_grad(oz, **bad) == -1


def test_norm_grad_limits_and_nothing_wanted(oz):
    assert norm_grad(oz, m=BIG) == -6
    assert norm_grad(oz, dX=N, dw=N, db=N) == norm_grad(oz, k=0) == 0
    assert norm_grad(oz, m=0, dX=N, flags=1) == 0


def xent(oz, m=4, n=8, k=8, type=BF16, X=16, ldx=8, W=16, ldw=8, ids=16, bits=64, scale=1.0, zl=0.0, loss=16, lse=16,
         picked=16):
    return oz.lib().oz2_linear_xent(m, n, k, type, X, ldx, W, ldw, ids, bits, scale, zl, loss, lse, picked, N)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(n=-1), dict(n=0), dict(k=-1), dict(type=F32), dict(type=E4M3), dict(bits=16), dict(ldx=7),
    dict(ldw=7), dict(X=N), dict(W=N), dict(ids=N), dict(loss=N), dict(lse=N), dict(picked=N), dict(X=17), dict(W=17),
    dict(ids=20), dict(loss=18), dict(lse=18), dict(picked=18), dict(scale=NAN), dict(scale=INF), dict(zl=NAN)])
def test_xent_refuses(oz, bad):
    assert xent(oz, **bad) == -1


def test_xent_limits_and_empty(oz):
    assert xent(oz, m=BIG) == xent(oz, n=BIG) == xent(oz, k=BIG, ldx=BIG, ldw=BIG) == -6
    assert xent(oz, m=0, X=N, ids=N, loss=N, lse=N, picked=N) == 0


def xent_grad(oz, m=4, n=8, k=8, type=BF16, dloss=16, X=16, ldx=8, W=16, ldw=8, ids=16, bits=64, lse=16, scale=1.0, zl=0.0,
              dX=16, lddx=8, dW=16, lddw=8, wt=BF16, flags=0):
    return oz.lib().oz2_linear_xent_grad(m, n, k, type, dloss, X, ldx, W, ldw, ids, bits, lse, scale, zl, dX, lddx, dW,
                                         lddw, wt, flags, N)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(n=0), dict(k=-1), dict(type=F32), dict(type=E4M3), dict(bits=16), dict(ldx=7), dict(ldw=7),
    dict(lddx=7), dict(lddw=7), dict(X=N), dict(W=N), dict(ids=N), dict(lse=N), dict(dloss=N), dict(dX=17), dict(dW=17),
    dict(wt=F32, dW=18), dict(wt=F16), dict(wt=E4M3), dict(flags=4), dict(flags=1), dict(dloss=18), dict(lse=18),
    dict(scale=INF), dict(zl=INF)])
def test_xent_grad_refuses(oz, bad):
    assert xent_grad(oz, **bad) == -1


def test_xent_grad_limits_and_nothing_wanted(oz):
    assert xent_grad(oz, m=BIG) == -6
    assert xent_grad(oz, dX=N, dW=N) == xent_grad(oz, k=0) == 0
    assert xent_grad(oz, m=0, wt=F32, flags=1, X=N, ids=N, lse=N, dloss=N) == 0


def distill(oz, m=4, n=8, k=8, top=4, type=BF16, X=16, ldx=8, W=16, ldw=8, ids=16, ldi=4, bits=64, T=16, ldt=4, tt=F32,
            temp=1.0, loss=16, lse=16, picked=16):
    return oz.lib().oz2_linear_distill(m, n, k, top, type, X, ldx, W, ldw, ids, ldi, bits, T, ldt, tt, temp, loss, lse,
                                       picked, N)


DISTILL = [dict(m=-1), dict(n=0), dict(k=-1), dict(top=0), dict(top=-1), dict(top=1025, ldi=2000, ldt=2000), dict(type=F32),
           dict(ldi=3), dict(ldt=3), dict(bits=16), dict(tt=E4M3), dict(temp=0.0), dict(temp=-1.0), dict(temp=NAN),
           dict(temp=1e-45), dict(ids=N), dict(T=N), dict(T=18), dict(ids=20), dict(X=N), dict(W=N), dict(lse=N)]


@pytest.mark.parametrize("bad", DISTILL + [dict(loss=N), dict(picked=N), dict(loss=18)])
def test_distill_refuses(oz, bad):
    assert distill(oz, **bad) == -1


def distill_grad(oz, m=4, n=8, k=8, top=4, type=BF16, dloss=16, X=16, ldx=8, W=16, ldw=8, ids=16, ldi=4, bits=64, T=16, ldt=4,
                 tt=F32, temp=1.0, lse=16, dX=16, lddx=8, dW=16, lddw=8, wt=BF16, flags=0):
    return oz.lib().oz2_linear_distill_grad(m, n, k, top, type, dloss, X, ldx, W, ldw, ids, ldi, bits, T, ldt, tt, temp, lse,
                                            dX, lddx, dW, lddw, wt, flags, N)


@pytest.mark.parametrize("bad", DISTILL + [dict(dloss=N), dict(wt=F16), dict(flags=1), dict(lddx=7), dict(lddw=7)])
def test_distill_grad_refuses(oz, bad):
    assert distill_grad(oz, **bad) == -1


def test_distill_limits_and_empty(oz):
    assert distill(oz, m=BIG) == distill_grad(oz, n=BIG) == -6
    assert distill(oz, m=0, X=N, ids=N, T=N, loss=N, lse=N, picked=N) == 0
    assert distill_grad(oz, dX=N, dW=N) == 0


def test_binding_refuses(oz):
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(6, 8, dtype=torch.bfloat16)
    ids, f = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    with pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_embedding(ids, w)
    with pytest.raises(AssertionError, match="int64 or int32"):
        oz.oz2_embedding(ids.float(), w)
    with pytest.raises(AssertionError, match="float32, bfloat16 or float16"):
        oz.oz2_embedding(ids, w.double())
    with pytest.raises(AssertionError, match="out has to be given"):
        oz.oz2_embedding_grad(x, ids, 6, accumulate=True)
    with pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_embedding_grad(x, ids, 6)
    with pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_layer_norm(x)
    with pytest.raises(AssertionError, match="float32, bfloat16 or float16"):
        oz.oz2_layer_norm(x.double())
    with pytest.raises(AssertionError, match="dy"):
        oz.oz2_layer_norm_grad(x.float(), x, f, f)
    with pytest.raises(AssertionError, match="one dtype"):
        oz.oz2_linear_xent(x, w.half(), ids)
    with pytest.raises(AssertionError, match="bfloat16 or float16"):
        oz.oz2_linear_xent(x.float(), w.float(), ids)
    with pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_linear_xent(x, w, ids)
    with pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_linear_xent_grad(f, x, w, ids, f)
    with pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_linear_distill(x, w, ids[:, None], f[:, None])


@pytest.mark.parametrize("what", ["table", "x", "weight", "bias", "head", "teacher"])
def test_a_lost_gradient_is_refused(oz, what):
    """Before anything else of the call is looked at (these are no CUDA tensors)."""
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(6, 8, dtype=torch.bfloat16)
    ids, v = torch.zeros(4, dtype=torch.int64), torch.zeros(8)
    t = torch.zeros(4, 2)
    (dict(table=w, x=x, weight=v, bias=v, head=w, teacher=t)[what]).requires_grad_()
    if what in ("weight", "bias"):
        call = lambda: oz.oz2_layer_norm(x, **{what: v})  # noqa: E731
    else:
        call = dict(table=lambda: oz.oz2_embedding(ids, w), x=lambda: oz.oz2_layer_norm(x),
                    head=lambda: oz.oz2_linear_xent(x, w, ids),
                    teacher=lambda: oz.oz2_linear_distill(x, w, torch.zeros(4, 2, dtype=torch.int64), t))[what]
    with pytest.raises(AssertionError, match="requires its gradient"):
        call()
    with torch.no_grad(), pytest.raises(AssertionError, match="CUDA"):
        call()


@pytest.mark.parametrize("what", ["embedding", "norm", "residual", "xent", "distill"])
def test_a_second_derivative_is_refused(oz, what):
    """A gradient that requires its own, before anything else of the call is looked at; x and weights
    that do are taken, up to the check of their device."""
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(6, 8, dtype=torch.bfloat16)
    ids, f = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    d = torch.zeros(4) if what in ("xent", "distill") else torch.zeros(4, 8, dtype=torch.bfloat16)
    x.requires_grad_()
    w.requires_grad_()
    call = dict(embedding=lambda: oz.oz2_embedding_grad(d, ids, 6), norm=lambda: oz.oz2_layer_norm_grad(d, x, f, f),
                residual=lambda: oz.oz2_layer_norm_grad(x.detach(), x, f, f, residual=d),
                xent=lambda: oz.oz2_linear_xent_grad(d, x, w, ids, f),
                distill=lambda: oz.oz2_linear_distill_grad(d, x, w, ids[:, None], f[:, None], f))[what]
    with pytest.raises(AssertionError, match="CUDA"):
        call()
    d.requires_grad_()
    with pytest.raises(AssertionError, match="requires its gradient"):
        call()
    with torch.no_grad(), pytest.raises(AssertionError, match="CUDA"):
        call()


def test_scales_that_pass_fp32_in_powers_of_two_are_refused(oz):
    """scale·log2 e is what multiplies the products: 3e38 is a number, that is not."""
    assert xent(oz, scale=3e38) == xent(oz, scale=-3e38) == xent_grad(oz, scale=3e38) == -1
    assert distill(oz, temp=1 / 3e38) == distill_grad(oz, temp=1 / 3e38) == -1
    assert xent(oz, m=0, scale=2e38) == 0
