"""Refusals of fira_embedding and fira_embedding_grad: arguments are checked before anything reaches the device."""
import pytest
import torch

from paper_2410_01623_b200 import binding as fb
from paper_2410_01623_b200 import build as fbuild

INVALID, SMALL = 1, 2
A, B, W, K = 1 << 20, 1 << 24, 1 << 28, 1 << 16        # made-up addresses: every case is refused before one is used


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fb.lib()


def lookup(lib, **change):
    a = dict(table=A, vocab=10, hidden=8, ld=0, dtype=0, tokens=K, bits=64, count=5, scale=1.0, out=B, ld_out=0)
    assert not set(change) - set(a)
    return lib.fira_embedding(*{**a, **change}.values(), None)


def grad(lib, **change):
    a = dict(tokens=K, bits=64, count=5, dY=A, ld=0, dtype=0, vocab=10, hidden=8, scale=1.0, G=B, ldg=0, grad_dtype=0,
             accumulate=0, work=W, work_bytes=1 << 30)
    assert not set(change) - set(a)
    return lib.fira_embedding_grad(*{**a, **change}.values(), None)


@pytest.mark.parametrize("change", [
    dict(vocab=0), dict(vocab=-1), dict(hidden=0), dict(count=-1), dict(count=(1 << 30) + 1), dict(vocab=(1 << 30) + 1),
    dict(hidden=(1 << 24) + 1), dict(bits=16), dict(dtype=2), dict(ld=7), dict(tokens=None), dict(tokens=K + 4)])
def test_bad_arguments_are_refused(lib, change):
    assert lookup(lib, **change) == INVALID
    assert len(lib.fira_last_error()) > 0
    assert grad(lib, **change) == INVALID


@pytest.mark.parametrize("change", [dict(table=None), dict(out=None), dict(ld_out=7), dict(table=A + 2), dict(out=B + 1)])
def test_bad_lookups_are_refused(lib, change):
    assert lookup(lib, **change) == INVALID


@pytest.mark.parametrize("change", [
    dict(dY=None), dict(G=None), dict(ldg=7), dict(grad_dtype=5), dict(dY=A + 2), dict(G=B + 2), dict(work=None),
    dict(work=W + 128)])
def test_bad_gradients_are_refused(lib, change):
    assert grad(lib, **change) == INVALID


@pytest.mark.parametrize("count,vocab,hidden", [(0, 1, 1), (1, 1, 1), (5, 10, 8), (4096, 32000, 512), (131072, 32000, 4096)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_small_workspaces_are_refused(lib, count, vocab, hidden, dtype):
    need = lib.fira_embedding_grad_work_bytes(count, vocab, hidden, dtype)
    assert need >= 8 * count + 4 * (vocab + 1)
    assert grad(lib, count=count, vocab=vocab, hidden=hidden, dtype=dtype, work_bytes=need - 1) == SMALL


def test_sizes_without_a_workspace(lib):
    assert lib.fira_embedding_grad_work_bytes(-1, 10, 8, 0) == 0
    assert lib.fira_embedding_grad_work_bytes(1, 0, 8, 0) == 0


def test_a_lookup_of_nothing_is_done(lib):
    assert lookup(lib, count=0, tokens=None, out=None) == 0


def test_binding_refuses_what_it_cannot_pass_on():
    tokens = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="int32 or int64"):
        fb.embedding(torch.zeros(4, 8), tokens.to(torch.int16))
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        fb.embedding(torch.zeros(4, 8, dtype=torch.float16), tokens)
    with pytest.raises(ValueError, match="matrix"):
        fb.embedding(torch.zeros(4), tokens)
    with pytest.raises(ValueError, match="strides"):
        fb.embedding(torch.zeros(8, 4).t(), tokens)
    with pytest.raises(ValueError, match="CUDA"):
        fb.embedding(torch.zeros(4, 8), tokens)
    with pytest.raises(ValueError, match="vocabulary"):
        fb.embedding_grad(tokens, torch.zeros(4, 8), 10)
    with pytest.raises(ValueError, match="out is needed"):
        fb.embedding_grad(tokens, torch.zeros(3, 8), 10, accumulate=True)
    with pytest.raises(ValueError, match="CUDA"):
        fb.embedding_grad(tokens, torch.zeros(3, 8), 10)
