"""Refusals of the Python functions that need no GPU."""
import pytest
import torch

from paper_2412_01034_b200 import api, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_check_workspace_refuses_what_is_no_workspace():
    with pytest.raises(ValueError):
        api.check_workspace(torch.zeros(64, dtype=torch.uint8))


def shapes():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    cache = dict(k_cache=bf(3, 2, 16, 64), v_cache=bf(3, 2, 16, 64), cu_q=i32(3), kv_len=i32(2), block_table=i32(2, 4))
    return {
        "rmsnorm": dict(x=bf(2, 8), weight=bf(8), residual=bf(2, 8), out=bf(2, 8), residual_out=bf(2, 8)),
        "rmsnorm_a8": dict(x=bf(2, 8), weight=bf(8), residual=bf(2, 8), out=bf(2, 8), residual_out=bf(2, 8)),
        "rope_append": dict(qkv=bf(2, 512), cos_sin=torch.zeros(4, 64), **cache, num_heads=4, out=bf(2, 4, 64)),
        "attn_paged": dict(q=bf(2, 4, 64), **cache, max_q_len=1, max_kv_len=16, out=bf(2, 4, 64), workspace=torch.zeros(1 << 20, dtype=torch.uint8)),
        "lora_batch_add": dict(x=bf(2, 8), a=bf(1, 8, 8), b=bf(1, 16, 8), y=bf(2, 16), cu_q=i32(2), adapter=i32(1), scales=torch.zeros(1), out=bf(2, 16),
                               workspace=torch.zeros(1 << 10, dtype=torch.uint8)),
    }


@pytest.mark.parametrize("op", list(shapes()))
def test_tensors_of_another_device_are_refused(op):
    """Each tensor in turn is on a device that is not the first one's: refused by name, before an address is taken."""
    args = shapes()[op]
    first = next(iter(args))
    for name, value in args.items():
        if name == first or not isinstance(value, torch.Tensor):
            continue
        with pytest.raises(ValueError, match=f"{name} is on meta, {first} on cpu"):
            getattr(api, op)(**dict(args, **{name: value.to("meta")}))
    with pytest.raises(ValueError, match="CUDA"):
        getattr(api, op)(**args)


A = 0x10000   # an aligned address that is never read


def test_sizes_near_32_bits_are_refused():
    """Where a kernel's counts would pass 2^31 the call is refused as a bad shape (on a machine without a GPU a launch would
    give another status)."""
    from paper_2412_01034_b200 import _lib
    lib, big = _lib.load(), 1 << 50
    assert lib.qil_rmsnorm(A, None, A, None, A, None, None, 0x7FFFFFFF, 8, 1e-5, None) == 2
    for n in (0x7FFFFFF8, 65535 * 128 + 8):
        assert lib.qil_lora_batch_add(A, A, A, A, A, A, A, A, 4, n, 32, 8, 2, 3, 32, n, n, A, big, None) == 2
    k = 0x7FFFFFF8
    assert lib.qil_lora_batch_add(A, A, A, A, A, A, A, A, 4, 16, k, 8, 2, 3, k, 16, 16, A, big, None) == 2
    sizes = (4, 2, 4, 2, 64, 128, 8, (1 << 24) - 1)
    assert lib.qil_rope_append(*[A] * 8, *sizes, 32, None) == 2
    assert lib.qil_attn_paged(*[A] * 7, *sizes, 4, 64, 0.1, A, big, None) == 2
    assert lib.qil_attn_paged_workspace_size(4, 2, 4, 2, 64, 4, 0x7FFFFFFF) >= lib.qil_attn_paged_workspace_size(4, 2, 4, 2, 64, 4, 1 << 30) > 0
