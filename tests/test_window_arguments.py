"""What the calls with a window, tree_norm_rope and the block-table calls refuse, without a GPU: the library checks its arguments
before anything is enqueued, the binding the shapes, types, strides and devices of its tensors."""
import ctypes
import importlib.machinery
import importlib.util
import os
import shutil

import numpy as np
import pytest
import torch

from paper_2604_09731_amd import binding as B

CTX = ctypes.create_string_buffer(4096)         # never looked into: every call below is refused before that
AT = 1 << 20                                    # an aligned address that nothing dereferences


def _prompt(window=5, sinks=1, **kw):
    p = B.PromptParams(dtype=B.SMART_BF16, batch=2, total_tokens=9, num_q_heads=8, num_kv_heads=2, head_dim=64, softmax_scale=0.125,
                       d_q=AT, d_k=AT, d_v=AT, q_stride=512, k_stride=128, v_stride=128, out_stride=512, d_cu_tokens=AT, d_out=AT)
    for name, value in kw.items():
        setattr(p, name, value)
    return B._lib().prompt_attention_window(CTX, None, ctypes.byref(p), window, sinks)


@pytest.mark.parametrize("bad", [dict(window=0), dict(window=-1), dict(window=-2 ** 31), dict(sinks=-1), dict(sinks=-2 ** 31), dict(dtype=2),
                                 dict(num_kv_heads=3), dict(head_dim=96), dict(softmax_scale=0.0), dict(q_stride=504), dict(k_stride=1 << 24),
                                 dict(d_q=None), dict(d_v=AT + 4), dict(d_cu_tokens=None), dict(batch=-1), dict(batch=1 << 23, k_stride=512, v_stride=512)])
def test_prompts_with_a_window(bad):
    assert _prompt(**bad) == B.SMART_EINVAL


def test_empty_prompts_are_no_error():
    assert _prompt(batch=0) == 0 and _prompt(total_tokens=0, d_q=None, d_cu_tokens=None) == 0
    assert _prompt(batch=0, window=0) == B.SMART_EINVAL
    assert B._lib().prompt_attention_window(None, None, None, 1, 0) == B.SMART_EINVAL


def _tree(window=5, sinks=1, **kw):
    p = B.TvaParams(dtype=B.SMART_BF16, kv_layout=B.SMART_KV_INTERLEAVED, batch=2, total_nodes=3, num_q_heads=8, num_kv_heads=2,
                    head_dim=64, block_size=16, max_blocks_per_seq=2, num_blocks=3, softmax_scale=0.1, d_q=AT, d_k_tree=AT, d_v_tree=AT,
                    d_k_cache=AT, d_v_cache=AT, cache_block_stride=2048, cache_head_stride=1024, d_block_table=AT, d_prefix_len=AT,
                    d_cu_nodes=AT, d_anc_mask=AT, d_out=AT)
    for name, value in kw.items():
        setattr(p, name, value)
    return B._lib().tree_verify_attention_window(CTX, None, ctypes.byref(p), window, sinks)


@pytest.mark.parametrize("bad", [dict(window=0), dict(window=-7), dict(sinks=-1), dict(dtype=7), dict(kv_layout=3), dict(head_dim=80),
                                 dict(block_size=12), dict(block_size=72), dict(num_q_heads=7), dict(softmax_scale=float("nan")), dict(d_q=None),
                                 dict(d_anc_mask=None), dict(d_block_table=None), dict(cache_head_stride=1000), dict(kv_cache_dtype=9),
                                 dict(kv_cache_dtype=B.SMART_FP8_E4M3), dict(kv_cache_dtype=B.SMART_FP4_E2M1, kv_layout=B.SMART_KV_PLAIN)])
def test_trees_with_a_window(bad):
    assert _tree(**bad) == B.SMART_EINVAL


def test_no_trees_are_no_error():
    assert B._lib().tree_verify_attention_window(None, None, None, 1, 0) == B.SMART_EINVAL


def _norm(**kw):
    p = B.NormRopeParams(dtype=B.SMART_BF16, n_tokens=3, num_q_heads=4, num_kv_heads=2, head_dim=64, rotary_dim=64, pairing=0, eps=1e-6,
                         base=1e4, d_position=AT, d_q=AT, d_k=2 * AT, d_q_out=3 * AT, d_k_out=4 * AT, q_stride=512, k_stride=512,
                         q_out_stride=256, k_out_stride=128)
    for name, value in kw.items():
        setattr(p, name, value)
    return B._lib().tree_norm_rope(CTX, None, ctypes.byref(p))


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(n_tokens=-1), dict(num_q_heads=-1), dict(num_q_heads=0, num_kv_heads=0), dict(num_kv_heads=65532, k_stride=1 << 23, k_out_stride=1 << 23),
                                 dict(head_dim=130), dict(head_dim=63), dict(head_dim=0), dict(rotary_dim=66), dict(rotary_dim=0), dict(rotary_dim=31),
                                 dict(pairing=2), dict(base=0.0), dict(base=float("nan")), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(eps=1e30), dict(eps=1e-40), dict(q_stride=255), dict(k_stride=127), dict(q_out_stride=255), dict(k_out_stride=64),
                                 dict(d_position=None), dict(d_q=None), dict(d_k=None), dict(d_q_out=None), dict(d_k_out=None), dict(d_q=AT + 1),
                                 dict(d_k_out=AT + 3), dict(d_q_weight=AT + 1), dict(dtype=B.SMART_F32, d_k_weight=AT + 2),
                                 dict(d_q_out=AT), dict(d_k_out=2 * AT)])
def test_norms_and_rotations(bad):
    assert _norm(**bad) == B.SMART_EINVAL


def test_no_tokens_are_no_error():
    assert _norm(n_tokens=0, d_q=None, d_position=None) == 0 and _norm(n_tokens=0, head_dim=63) == B.SMART_EINVAL
    assert B._lib().tree_norm_rope(None, None, None) == B.SMART_EINVAL


_EXTEND = dict(batch=2, bs=16, width=4, nb=9, length=AT, new=2 * AT, held=3 * AT, free=4 * AT, cap=5, count=5 * AT, table=6 * AT, rows=7, cu=7 * AT,
               slots=8 * AT, new_length=9 * AT, new_held=10 * AT, new_count=11 * AT, status=12 * AT)
_RELEASE = dict(batch=2, bs=16, width=4, window=8, sinks=1, length=AT, held=2 * AT, released=3 * AT, done=None, table=4 * AT, free=5 * AT, cap=5,
                count=6 * AT, new_length=7 * AT, new_held=8 * AT, new_released=9 * AT, new_count=10 * AT, status=11 * AT)


def _extend(**kw):
    return B._lib().kv_cache_extend(CTX, None, *dict(_EXTEND, **kw).values())


def _release(**kw):
    return B._lib().kv_cache_release(CTX, None, *dict(_RELEASE, **kw).values())


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(batch=(1 << 30) + 1), dict(bs=0), dict(bs=-16), dict(width=-1), dict(width=1 << 28), dict(nb=-1), dict(cap=-1), dict(rows=-1),
                                 dict(rows=1 << 31), dict(length=None), dict(new=None), dict(held=None), dict(free=None), dict(count=None),
                                 dict(table=None), dict(cu=None), dict(slots=None), dict(new_length=None), dict(new_held=None), dict(new_count=None),
                                 dict(status=None), dict(new_count=5 * AT), dict(new_length=AT), dict(new_held=3 * AT), dict(status=2 * AT), dict(cu=AT)])
def test_extending(bad):
    assert _extend(**bad) == B.SMART_EINVAL


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(batch=(1 << 30) + 1), dict(bs=0), dict(width=-1), dict(width=1 << 28), dict(window=-1), dict(sinks=-1),
                                 dict(window=0, sinks=1), dict(cap=-1), dict(length=None), dict(held=None), dict(released=None), dict(table=None),
                                 dict(free=None), dict(count=None), dict(new_length=None), dict(new_held=None), dict(new_released=None),
                                 dict(new_count=None), dict(status=None), dict(new_count=6 * AT), dict(new_length=AT), dict(new_held=2 * AT),
                                 dict(new_released=3 * AT), dict(done=7 * AT)])
def test_releasing(bad):
    assert _release(**bad) == B.SMART_EINVAL


# ---- the binding's side ------------------------------------------------------------------------------------------------------
@pytest.fixture()
def native(tmp_path):
    """A copy of the module with state of its own, whose entry points count how often they are called."""
    path = shutil.copy(os.path.join(os.path.dirname(B.__file__), "_marshal.so"), tmp_path / "_marshal.so")
    loader = importlib.machinery.ExtensionFileLoader("_marshal", str(path))
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader))
    called = []
    entry = ctypes.CFUNCTYPE(ctypes.c_int32)(lambda: called.append(1) or 0)
    address = ctypes.cast(entry, ctypes.c_void_p).value
    module.setup((address,) * len(B._NATIVE_ENTRIES), None, lambda: 0, lambda device: 0)
    return module, called, entry


Q, KV = torch.zeros(9, 8, 64), torch.zeros(9, 2, 64)
CU, I32 = torch.tensor([0, 4, 9], dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
POS, TABLE, MASK = torch.zeros(9, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(9, 2, dtype=torch.int64)
CACHE, W, ONE = torch.zeros(3, 2, 16, 64), torch.zeros(64), torch.zeros(1, dtype=torch.int32)
SKIP = torch.zeros(4, dtype=torch.int32)[::2]
CALLS = {
    "prompt_window": [0, Q, KV, KV, CU, 0.1, None, None, True, 5, 1],
    "attention_window": [0, Q, KV, KV, CACHE, CACHE, TABLE, I32, CU, MASK, 0.1, 0, 16, None, None, False, 0, None, None, False, None, 5, 1, False],
    "norm_rope": [0, POS, Q, KV, W, W, 1e-6, 1e4, None, 0, None, None],
    "cache_extend": [0, I32, I32, I32, TABLE, POS, ONE, 16, 9, 20],
    "cache_release": [0, I32, I32, I32, TABLE, POS, ONE, 16, I32, 5, 1],
}
BAD = {
    "prompt_window": [(1, Q.double()), (2, KV[:8]), (4, CU.long()), (6, Q[:8]), (9, 1.5), (9, "5"), (9, 2 ** 31), (10, None), (10, -2 ** 40)],
    "attention_window": [(1, Q.bfloat16()), (2, KV[:8]), (3, torch.zeros(9, 4, 64)[:, ::2]), (4, CACHE.double()), (4, CACHE[:2]), (5, CACHE.bfloat16()),
                         (4, torch.zeros(3, 4, 16, 64)), (6, TABLE.long()), (6, TABLE[:1]), (7, I32[:1]), (8, CU.long()), (9, MASK.int()), (13, Q[:8]),
                         (20, I32[:1]), (21, 2.0), (21, None), (22, 2 ** 33)],
    "norm_rope": [(1, POS.long()), (1, POS[:8]), (2, Q.double()), (2, Q[0]), (2, Q.bfloat16()), (3, KV[:8]), (3, KV[..., :32]), (4, W.bfloat16()),
                  (4, W[:63]), (5, torch.zeros(128)[::2]), (2, torch.zeros(9, 64, 8).transpose(1, 2)), (8, 2.0), (9, None), (10, Q[:8]),
                  (11, KV.bfloat16()), (10, torch.zeros(9, 16, 64)[:, ::2])],
    "cache_extend": [(1, I32.long()), (2, I32[:1]), (3, SKIP.long()), (1, SKIP), (4, TABLE.long()), (4, TABLE[:1]), (4, POS), (5, POS.long()), (6, torch.zeros(0, dtype=torch.int32)),
                     (7, 16.0), (8, None), (9, -1), (9, 2 ** 31)],
    "cache_release": [(1, I32.long()), (2, I32[:1]), (3, None), (4, TABLE[:1]), (5, POS.long()), (6, POS.long()), (8, I32.bool()), (8, I32[:1]),
                      (9, 1.0), (10, None), (9, 2 ** 31)],
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_binding_refuses(name, native):
    module, called, entry = native          # (entry: kept alive)
    call = getattr(module, name)
    call(*CALLS[name])
    assert called.pop() and not called
    for at, wrong in BAD[name]:
        args = list(CALLS[name])
        args[at] = wrong
        with pytest.raises((ValueError, TypeError, RuntimeError, IndexError, AssertionError)):
            call(*args)
        assert not called, (at, wrong)
    with pytest.raises(TypeError):
        call(*CALLS[name][:-1])


def test_what_the_handle_refuses():
    lib = object.__new__(B.SmartTree)
    lib._native, lib._h, lib.device = None, None, 0
    for call in (lambda: lib.prompt_attention(Q, KV, KV, CU, 0.1, window=3), lambda: lib.tree_norm_rope(POS, Q, KV, W, W),
                 lambda: lib.kv_cache_extend(I32, I32, I32, TABLE, POS, ONE, 16, 9, 20), lambda: lib.kv_cache_release(I32, I32, I32, TABLE, POS, ONE, 16),
                 lambda: lib.tree_verify_attention(Q, KV, KV, CACHE, CACHE, TABLE, I32, CU, MASK, 0.1, 0, window=3)):
        with pytest.raises(ValueError):         # (tensors that are not on its GPU)
            call()
    lib.device = -1                             # where these tensors are
    with pytest.raises(ValueError):
        lib.prompt_attention(Q, KV, KV, CU, 0.1, sinks=3)
    with pytest.raises(ValueError):
        lib.tree_verify_attention(Q, KV, KV, CACHE, CACHE, TABLE, I32, CU, MASK, 0.1, 0, sinks=3)
    with pytest.raises(ValueError):
        lib.tree_verify_attention(Q, KV, KV, CACHE, CACHE, TABLE, I32, CU, MASK, 0.1, 0, window=3, static=True)


def test_numpy_integers_are_integers(native):
    module, called, entry = native
    args = list(CALLS["prompt_window"])
    args[9], args[10] = np.int64(5), np.int32(1)
    module.prompt_window(*args)
    assert called.pop()
