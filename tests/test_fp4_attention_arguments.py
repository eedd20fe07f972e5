"""What the binding refuses of attention over a 4-bit cache beside the caches' pages, without a GPU: every tensor's element type,
shape, layout and device is looked at before its address goes to the library."""
import pytest
import torch

from paper_2604_09731_amd import binding as B
from tests.test_fp4_prompt_arguments import CACHE, CALLS, CU, I32, KV, Q, native  # noqa: F401  (native: a fixture)

TABLE, MASK = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(9, 2, dtype=torch.int64)
# position in the call, and what it must not be
BAD = [(1, Q.bfloat16()), (1, torch.zeros(9, 16, 64)[:, ::2]), (1, torch.zeros(10, 8, 64)), (1, torch.zeros(9, 8, 32)),
       (2, KV[:8]), (2, KV.bfloat16()), (2, KV[..., :32].contiguous()), (2, torch.zeros(9, 4, 64)[:, ::2]), (2, KV[0]),
       (3, KV[:8]), (3, torch.zeros(9, 4, 64)), (3, torch.zeros(9, 4, 64)[:, ::2]), (3, KV.bfloat16()),
       (6, TABLE.long()), (6, TABLE[:1]), (6, torch.zeros(2, 6, dtype=torch.int32)[:, ::2]), (6, None),
       (7, I32.long()), (7, I32[:1]), (7, torch.zeros(4, dtype=torch.int32)[::2]),
       (8, CU.long()), (8, CU.view(3, 1)), (8, torch.zeros(6, dtype=torch.int32)[::2]), (8, CU[:0]),
       (9, MASK.int()), (9, MASK[:8]), (9, torch.zeros(9, 4, dtype=torch.int64)[:, ::2]),
       (13, Q[:8]), (13, Q.bfloat16()), (13, torch.zeros(9, 16, 64)[:, ::2]),
       (14, torch.zeros(9, 7)), (14, torch.zeros(9, 8, dtype=torch.float64)), (14, torch.zeros(9, 16)[:, ::2]),
       (20, I32.long()), (20, I32[:1])]
BAD += [(at, t.to("meta")) for at, t in ((1, Q), (2, KV), (4, CACHE), (5, CACHE), (6, TABLE), (7, I32), (8, CU), (9, MASK), (13, Q),
                                         (14, torch.zeros(9, 8)), (20, I32))]


@pytest.mark.parametrize("at,wrong", BAD)
def test_attention_over_a_4_bit_cache_refuses_tensors(native, at, wrong):  # noqa: F811
    module, called, entry = native
    args = list(CALLS["attention_fp4"])
    args[at] = wrong
    with pytest.raises((ValueError, TypeError, IndexError)):
        module.attention_fp4(*args)
    assert not called


def test_attention_over_a_4_bit_cache_takes_all_that_fits(native):  # noqa: F811
    module, called, entry = native
    args = list(CALLS["attention_fp4"])
    args[2], args[3] = torch.zeros(12, 2, 64), torch.zeros(12, 2, 64)        # rows beyond the call's
    args[13], args[14], args[20] = torch.zeros_like(Q), torch.zeros(9, 8), torch.zeros(2, dtype=torch.int32)
    out, lse = module.attention_fp4(*args)
    assert called.pop() and out.data_ptr() == args[13].data_ptr() and lse.data_ptr() == args[14].data_ptr()
    args[4] = args[5] = args[6] = None                                      # no cached prefix
    module.attention_fp4(*args)
    assert called.pop()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.int8])
def test_a_cache_said_to_hold_fp8_that_holds_something_else_is_refused(dtype):
    called = []
    lib = object.__new__(B.SmartTree)
    lib._native, lib._h, lib.device = type("native", (), {"attention": lambda *a: called.append(a)}), None, 0
    cache = torch.zeros(3, 2, 16, 64, dtype=dtype)
    with pytest.raises(ValueError):
        lib.tree_verify_attention(Q, KV, KV, cache, cache, TABLE, I32, CU, MASK, 0.1, B.SMART_KV_PLAIN, k_scale=1.0, v_scale=1.0,
                                  kv_cache_dtype=B.SMART_FP8_E4M3)
    assert not called
    bytes_ = cache.to(torch.uint8)
    lib.tree_verify_attention(Q, KV, KV, bytes_, bytes_, TABLE, I32, CU, MASK, 0.1, B.SMART_KV_PLAIN, k_scale=1.0, v_scale=1.0,
                              kv_cache_dtype=B.SMART_FP8_E4M3)
    assert len(called) == 1
