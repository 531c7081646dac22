"""Host-side refusals of the operators between the linears of a decoder layer (no GPU needed)."""
import math

import pytest
import torch

from paper_2412_01034_b200 import _lib, api, build

A, U = 0x10000, 0x10008   # an aligned address that is never read, and one off 16 bytes


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def test_rmsnorm_validation(lib):
    f = lambda x=A, r=None, w=A, ro=None, y=A, q=None, s=None, M=2, K=16, eps=1e-5: lib.qil_rmsnorm(x, r, w, ro, y, q, s, M, K, eps, None)  # noqa: E731
    for kw in (dict(x=None), dict(w=None), dict(y=None), dict(q=A), dict(ro=A)):
        assert f(**kw) == 1, kw
    for kw in (dict(M=0), dict(K=0), dict(K=12), dict(K=-8)):
        assert f(**kw) == 2, kw
    for kw in (dict(x=U), dict(r=U), dict(w=U), dict(y=U), dict(q=U, s=A), dict(q=A, s=0x10002), dict(r=A, ro=U)):
        assert f(**kw) == 3, kw
    for kw in (dict(K=32776), dict(eps=-1.0), dict(eps=math.nan)):
        assert f(**kw) == 4, kw


def paged(f, order):
    base = dict(total_q=4, num_seqs=2, num_heads=4, num_kv_heads=2, head_dim=64, page_size=16, num_pages=8, max_pages=4)
    shape = [("total_q", 0), ("num_seqs", 0), ("num_heads", 0), ("num_kv_heads", 0), ("num_pages", 0), ("max_pages", 0),
             ("num_kv_heads", 3), ("max_pages", 1 << 28), ("num_pages", 1 << 27), ("total_q", 1 << 30)]
    unsupported = [("head_dim", 96), ("head_dim", 0), ("page_size", 8), ("page_size", 48), ("page_size", 256)]
    for code, changes in ((2, shape), (4, unsupported)):
        for name, value in changes:
            assert f([dict(base, **{name: value})[n] for n in order]) == code, (name, value)
    return [base[n] for n in order]


ORDER = ["total_q", "num_seqs", "num_heads", "num_kv_heads", "head_dim", "page_size", "num_pages", "max_pages"]


def test_rope_append_validation(lib):
    sizes = paged(lambda s: lib.qil_rope_append(*[A] * 8, *s, 32, None), ORDER)
    for i in range(8):
        p = [A] * 8
        p[i] = None
        assert lib.qil_rope_append(*p, *sizes, 32, None) == 1
        p[i] = U if i < 5 else 0x10002
        assert lib.qil_rope_append(*p, *sizes, 32, None) == 3
    assert lib.qil_rope_append(*[A] * 8, *sizes, 0, None) == 2


def test_attn_paged_validation(lib):
    big = 1 << 40
    sizes = paged(lambda s: lib.qil_attn_paged(*[A] * 7, *s, 4, 64, 0.1, A, big, None), ORDER)
    for i in range(7):
        p = [A] * 7
        p[i] = None
        assert lib.qil_attn_paged(*p, *sizes, 4, 64, 0.1, A, big, None) == 1
        p[i] = U if i < 4 else 0x10002
        assert lib.qil_attn_paged(*p, *sizes, 4, 64, 0.1, A, big, None) == 3
    assert lib.qil_attn_paged(*[A] * 7, *sizes, 0, 64, 0.1, A, big, None) == 2
    assert lib.qil_attn_paged(*[A] * 7, *sizes, 4, 0, 0.1, A, big, None) == 2
    for bad in (math.nan, math.inf):
        assert lib.qil_attn_paged(*[A] * 7, *sizes, 4, 64, bad, A, big, None) == 4
    need = lib.qil_attn_paged_workspace_size(4, 2, 4, 2, 64, 4, 64)
    assert need > 0
    assert lib.qil_attn_paged(*[A] * 7, *sizes, 4, 64, 0.1, A, need - 1, None) == 5
    assert lib.qil_attn_paged(*[A] * 7, *sizes, 4, 64, 0.1, None, big, None) == 5
    assert lib.qil_attn_paged(*[A] * 7, *sizes, 4, 64, 0.1, U, big, None) == 3
    for bad in ((0, 2, 4, 2, 64, 4, 64), (4, 0, 4, 2, 64, 4, 64), (4, 2, 4, 3, 64, 4, 64), (4, 2, 4, 2, 64, 0, 64), (4, 2, 4, 2, 64, 4, 0)):
        assert lib.qil_attn_paged_workspace_size(*bad) == 0


def test_lora_batch_validation(lib):
    base = dict(M=4, N=16, K=32, rank=8, num_seqs=2, num_adapters=3, ldx=32, ldy=16, ldo=16)
    big = 1 << 40
    out = 0x20000

    def f(p=(A, A, A, A, out, A, A, A), ws=A, nbytes=big, **kw):
        return lib.qil_lora_batch_add(*p, *dict(base, **kw).values(), ws, nbytes, None)

    for i in range(8):
        p = [A, A, A, A, out, A, A, A]
        p[i] = None
        assert f(p) == 1
        p[i] = U if i < 5 else 0x10002
        assert f(p) == 3
    for kw in (dict(M=0), dict(N=0), dict(K=0), dict(rank=0), dict(num_seqs=0), dict(num_adapters=0), dict(N=12), dict(K=36), dict(rank=12),
               dict(ldx=24), dict(ldx=36), dict(ldy=8), dict(ldo=8), dict(ldo=20), dict(N=1 << 28, ldy=1 << 28, ldo=1 << 28)):
        assert f(**kw) == 2, kw
    assert f((A, A, A, A, A, A, A, A), ldo=24) == 2      # in place with another stride
    assert f(rank=72) == 4
    need = lib.qil_lora_batch_workspace_size(4, 2, 8)
    assert need > 0 and f(nbytes=need - 1) == 5 and f(ws=None) == 5 and f(ws=U) == 3
    assert lib.qil_lora_batch_workspace_size(0, 1, 8) == 0
    assert f(num_seqs=(1 << 24) + 1) == 2 and f(M=(1 << 30) + 1) == 2


def test_the_binding_refuses_wrong_tensors():
    """Types, shapes and layouts are looked at before an address is taken (CPU tensors: nothing can be launched)."""
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="x is torch.float32"):
        api.rmsnorm(torch.zeros(2, 8), bf(8))
    with pytest.raises(ValueError, match="contiguous CUDA tensor"):
        api.rmsnorm(bf(2, 8), bf(8))
    with pytest.raises(ValueError, match="expected bfloat16"):
        api.lora_batch_add(torch.zeros(2, 8), bf(1, 8, 8), bf(1, 8, 8), bf(2, 8), i32(2), i32(1), torch.zeros(1))
    with pytest.raises(ValueError):
        api.lora_batch_add(bf(2, 16), bf(1, 8, 8), bf(1, 8, 8), bf(2, 8), i32(2), i32(1), torch.zeros(1))
    with pytest.raises(ValueError):
        api.attn_paged(bf(2, 4, 64), bf(3, 2, 16, 64), bf(3, 2, 16, 64), i32(3), torch.zeros(2), i32(2, 4), 1, 16)
    with pytest.raises(ValueError):
        api.rope_append(bf(2, 100), torch.zeros(4, 64), bf(3, 2, 16, 64), bf(3, 2, 16, 64), i32(3), i32(2), i32(2, 4), 4)
