"""Host-side refusals of the quantised cache's operators (no GPU needed)."""
import math

import pytest
import torch

from paper_2412_01034_b200 import _lib, api, build
from tests.test_abi_layer import ORDER, A, U, paged

BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def test_rope_append_q_validation(lib):
    f = lambda s, p=(A,) * 10, bits=8, pos=32: lib.qil_rope_append_q(*p[:7], bits, *p[7:], *s, pos, None)  # noqa: E731
    sizes = paged(f, ORDER)
    for i in range(10):
        p = [A] * 10
        p[i] = None
        assert f(sizes, p) == 1
        p[i] = U if i < 7 else 0x10002
        assert f(sizes, p) == 3
    assert f(sizes, pos=0) == 2
    for bits in (0, 2, 5, 16):
        assert f(sizes, bits=bits) == 4


def test_kv_read_q_validation(lib):
    order = [n for n in ORDER if n != "num_heads"]
    f = lambda s, p=(A,) * 9, bits=4: lib.qil_kv_read_q(*p[:4], bits, *p[4:], *s, None)  # noqa: E731
    sizes = dict(total_q=4, num_seqs=2, num_kv_heads=2, head_dim=64, page_size=16, num_pages=8, max_pages=4)
    for name in ("total_q", "num_seqs", "num_kv_heads", "num_pages", "max_pages"):
        assert f([dict(sizes, **{name: 0})[n] for n in order]) == 2
    for name, value in (("head_dim", 96), ("page_size", 8), ("page_size", 256)):
        assert f([dict(sizes, **{name: value})[n] for n in order]) == 4
    s = [sizes[n] for n in order]
    for i in range(9):
        p = [A] * 9
        p[i] = None
        assert f(s, p) == 1
        p[i] = U if i < 6 else 0x10002
        assert f(s, p) == 3
    assert f(s, bits=3) == 4


def test_attn_paged_q_validation(lib):
    f = lambda s, p=(A,) * 9, bits=8, mq=4, mkv=64, scale=0.1, ws=A, n=BIG: lib.qil_attn_paged_q(*p[:5], bits, *p[5:], *s, mq, mkv, scale, ws, n, None)  # noqa: E731
    sizes = paged(f, ORDER)
    for i in range(9):
        p = [A] * 9
        p[i] = None
        assert f(sizes, p) == 1
        p[i] = U if i < 6 else 0x10002
        assert f(sizes, p) == 3
    assert f(sizes, mq=0) == 2 and f(sizes, mkv=0) == 2 and f(sizes, bits=16) == 4
    for bad in (math.nan, math.inf):
        assert f(sizes, scale=bad) == 4
    for bits in (4, 8):
        need = lib.qil_attn_paged_q_workspace_size(4, 2, 4, 2, 64, bits, 4, 64)
        assert need > 0 and f(sizes, bits=bits, n=need - 1) == 5 and f(sizes, bits=bits, ws=None) == 5
    assert f(sizes, ws=U) == 3
    for bad in ((0, 2, 4, 2, 64, 8, 4, 64), (4, 0, 4, 2, 64, 8, 4, 64), (4, 2, 4, 3, 64, 8, 4, 64), (4, 2, 4, 2, 64, 6, 4, 64), (4, 2, 4, 2, 64, 8, 0, 64)):
        assert lib.qil_attn_paged_q_workspace_size(*bad) == 0


def bf(*s):
    return torch.zeros(s, dtype=torch.bfloat16)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def calls(bits):
    cache = api.new_kv_cache_q(3, 2, 16, 64, bits, device="cpu")
    after = dict(kv_len=i32(2), block_table=i32(2, 4))
    return {
        "rope_append_q": dict(qkv=bf(2, 512), cos_sin=torch.zeros(4, 64), cache=cache, cu_q=i32(3), **after, num_heads=4, out=bf(2, 4, 64)),
        "kv_read_q": dict(cache=cache, cu=i32(3), **after, total_rows=2, out=(bf(2, 2, 64), bf(2, 2, 64))),
        "attn_paged_q": dict(q=bf(2, 4, 64), cache=cache, cu_q=i32(3), **after, max_q_len=1, max_kv_len=16, out=bf(2, 4, 64),
                             workspace=torch.zeros(1 << 20, dtype=torch.uint8)),
    }


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("op", list(calls(8)))
def test_the_binding_refuses_wrong_tensors(op, bits):
    """Types, shapes and devices are looked at before an address is taken (CPU tensors: nothing can be launched)."""
    args = calls(bits)[op]
    f = getattr(api, op)
    with pytest.raises(ValueError, match="CUDA"):
        f(**args)
    cache = args["cache"]
    wrong = [cache._replace(k=cache.k.float()), cache._replace(v=cache.v[:2]), cache._replace(v=cache.v.to(torch.int16)),
             cache._replace(k_scale=cache.k_scale.float()), cache._replace(v_scale=cache.v_scale[:, :1]), cache._replace(k_scale=cache.k_scale[..., None])]
    for c in wrong:
        with pytest.raises(ValueError):
            f(**dict(args, cache=c))
    for field in ("v", "k_scale", "v_scale"):
        with pytest.raises(ValueError, match="meta"):
            f(**dict(args, cache=cache._replace(**{field: getattr(cache, field).to("meta")})))
    for name in ("kv_len", "block_table", "cu" if op == "kv_read_q" else "cu_q"):
        with pytest.raises(ValueError):
            f(**dict(args, **{name: args[name].long()}))
        with pytest.raises(ValueError, match="meta"):
            f(**dict(args, **{name: args[name].to("meta")}))


def test_a_cache_of_other_bits_is_refused():
    with pytest.raises(api.QilError):
        api.new_kv_cache_q(3, 2, 16, 64, bits=16, device="cpu")
    assert api.new_kv_cache_q(3, 2, 16, 64, bits=4, device="cpu").bits == 4 and api.new_kv_cache_q(3, 2, 16, 64, device="cpu").bits == 8
