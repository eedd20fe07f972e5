"""What prompt_attention and the 4-bit cache's calls refuse, without a GPU: the library checks its arguments before anything is
enqueued, the binding the shapes, types and strides of its tensors."""
import ctypes
import importlib.machinery
import importlib.util
import os
import shutil
import types

import pytest
import torch

from paper_2604_09731_amd import binding as B

CTX = ctypes.create_string_buffer(4096)         # never looked into: every call below is refused before that
AT = 1 << 20                                    # an aligned address that nothing dereferences


def _prompt(**kw):
    p = B.PromptParams(dtype=B.SMART_BF16, batch=2, total_tokens=9, num_q_heads=8, num_kv_heads=2, head_dim=64, softmax_scale=0.125,
                       d_q=AT, d_k=AT, d_v=AT, q_stride=512, k_stride=128, v_stride=128, out_stride=512, d_cu_tokens=AT, d_out=AT)
    for name, value in kw.items():
        setattr(p, name, value)
    return B._lib().prompt_attention(CTX, None, ctypes.byref(p))


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(batch=-1), dict(total_tokens=-1), dict(num_q_heads=0), dict(num_kv_heads=0), dict(num_kv_heads=3),
    dict(head_dim=96), dict(head_dim=0), dict(softmax_scale=0.0), dict(softmax_scale=float("nan")), dict(softmax_scale=1e30),
    dict(total_tokens=1 << 28), dict(q_stride=504), dict(out_stride=511), dict(k_stride=127), dict(v_stride=64), dict(k_stride=1 << 24), dict(v_stride=1 << 24),
    dict(q_stride=516), dict(k_stride=132), dict(v_stride=129), dict(out_stride=1028), dict(d_q=None), dict(d_k=None),
    dict(d_v=None), dict(d_out=None), dict(d_cu_tokens=None), dict(d_q=AT + 8), dict(d_k=AT + 2), dict(d_v=AT + 4), dict(d_out=AT + 8),
])
def test_prompt_attention_refuses(bad):
    assert _prompt(**bad) == B.SMART_EINVAL


def test_empty_prompts_are_no_error():
    assert _prompt(batch=0) == 0 and _prompt(total_tokens=0) == 0
    assert _prompt(total_tokens=0, d_q=None, d_k=None, d_v=None, d_out=None, d_cu_tokens=None) == 0
    assert B._lib().prompt_attention(None, None, None) == B.SMART_EINVAL


PAGE = B.fp4_page_bytes(16, 64)
_WRITE = dict(src=B.SMART_BF16, n=5, heads=2, D=64, bs=16, nb=3, a=AT, b=AT, slots=AT, k=AT, v=AT, block=2 * PAGE, head=PAGE)


def _write(**kw):
    c = dict(_WRITE, **kw)
    return B._lib().kv_cache_write_fp4(CTX, None, c["src"], c["n"], c["heads"], c["D"], c["bs"], c["nb"], c["a"], c["b"], c["slots"],
                                       c["k"], c["v"], c["block"], c["head"])


def _read(**kw):
    c = dict(_WRITE, **kw)
    return B._lib().kv_cache_read_fp4(CTX, None, c["src"], c["n"], c["heads"], c["D"], c["bs"], c["nb"], c["k"], c["v"], c["block"],
                                      c["head"], c["slots"], c["a"], c["b"])


def _commit(**kw):
    c = dict(_WRITE, depth=4, blocks=3, cu=AT, length=AT, path=AT, table=AT, prefix=AT, new=2 * AT, status=AT, **{})
    c.update(kw)
    return B._lib().tree_commit_fp4(CTX, None, c["src"], c["n"], c["depth"], c["heads"], c["D"], c["bs"], c["blocks"], c["nb"], c["cu"],
                                    c["length"], c["path"], c["a"], c["b"], c["table"], c["prefix"], c["k"], c["v"], c["block"],
                                    c["head"], c["new"], c["status"])


_PAGES = [dict(src=2), dict(n=-1), dict(heads=0), dict(D=48), dict(D=0), dict(bs=12), dict(bs=0), dict(nb=-1), dict(head=PAGE - 16),
          dict(head=PAGE + 8, block=4 * PAGE), dict(block=PAGE - 16), dict(block=2 * PAGE + 4), dict(k=AT + 8), dict(v=AT + 1),
          dict(k=None), dict(v=None), dict(a=None), dict(b=None), dict(a=AT + 2), dict(b=AT + 8)]


@pytest.mark.parametrize("bad", _PAGES + [dict(slots=None)])
def test_writing_and_reading_refuse(bad):
    assert _write(**bad) == B.SMART_EINVAL
    assert _read(**bad) == B.SMART_EINVAL


@pytest.mark.parametrize("bad", _PAGES + [dict(depth=-1), dict(depth=129), dict(blocks=-1), dict(n=65536), dict(cu=None),
                                          dict(length=None), dict(path=None), dict(table=None), dict(prefix=None), dict(new=None),
                                          dict(status=None), dict(new=AT)])
def test_commit_refuses(bad):
    assert _commit(**bad) == B.SMART_EINVAL


def test_nothing_to_do_is_no_error():
    assert _write(n=0) == 0 and _read(n=0) == 0 and _commit(n=0) == 0


def _attention(**kw):
    p = B.TvaParams(dtype=B.SMART_BF16, kv_layout=B.SMART_KV_INTERLEAVED, batch=2, total_nodes=0, num_q_heads=8, num_kv_heads=2,
                    head_dim=64, block_size=16, max_blocks_per_seq=2, num_blocks=3, softmax_scale=0.1,
                    kv_cache_dtype=B.SMART_FP4_E2M1, d_k_cache=AT, d_v_cache=AT, cache_block_stride=2 * PAGE, cache_head_stride=PAGE)
    for name, value in kw.items():
        setattr(p, name, value)
    return B._lib().tree_verify_attention(CTX, None, ctypes.byref(p))


@pytest.mark.parametrize("bad", [dict(kv_layout=B.SMART_KV_PLAIN, cache_token_stride=64), dict(cache_head_stride=PAGE - 16),
                                 dict(cache_head_stride=PAGE + 4), dict(cache_block_stride=2 * PAGE + 8), dict(d_k_cache=AT + 8),
                                 dict(d_v_cache=AT + 4), dict(kv_cache_dtype=4), dict(kv_cache_dtype=1), dict(block_size=12)])
def test_attention_over_a_4_bit_cache_refuses(bad):
    assert _attention(**bad) == B.SMART_EINVAL


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
CU = torch.tensor([0, 4, 9], dtype=torch.int32)
CACHE = torch.zeros(3, 2, PAGE, dtype=torch.uint8)
SLOTS = torch.zeros(9, dtype=torch.int64)
I32 = torch.zeros(2, dtype=torch.int32)
FUSED = torch.zeros(9, 12, 64)                  # q, k and v of one projection
CALLS = {
    "prompt": [0, Q, KV, KV, CU, 0.1, None, None, True],
    "cache_write_fp4": [0, KV, KV, SLOTS, CACHE, CACHE, 16],
    "cache_read_fp4": [0, SLOTS, CACHE, CACHE, 16, KV, KV],
    "commit_fp4": [0, CU, I32, torch.zeros(2, 5, dtype=torch.int32), KV, KV, CACHE, CACHE, torch.zeros(2, 3, dtype=torch.int32), I32, 16],
    "attention_fp4": [0, Q, KV, KV, CACHE, CACHE, torch.zeros(2, 3, dtype=torch.int32), I32, CU, torch.zeros(9, 2, dtype=torch.int64),
                      0.1, 1, 16, None, None, False, 0, None, None, False, None],
}
BAD = {
    "prompt": [(1, Q.double()), (1, Q[0]), (1, Q.bfloat16()), (2, KV[:8]), (3, KV[:8]), (2, KV[..., :32]), (3, torch.zeros(9, 4, 64)),
               (1, torch.zeros(9, 64, 8).transpose(1, 2)), (2, torch.zeros(9, 4, 64)[:, ::2]), (4, CU.long()), (4, CU.view(3, 1)),
               (4, torch.zeros(6, dtype=torch.int32)[::2]), (6, Q[:8]), (6, Q.bfloat16()), (7, torch.zeros(9, 7)),
               (7, torch.zeros(9, 8, dtype=torch.float64)), (1, None), (5, "x")],
    "cache_write_fp4": [(1, KV[:8]), (1, torch.zeros(9, 4, 64)[:, ::2]), (2, KV.bfloat16()), (3, SLOTS.int()), (3, SLOTS[:8]), (4, CACHE[:2]),
                        (4, CACHE.view(torch.int8)), (4, CACHE[..., :-16]), (5, torch.zeros(3, 4, PAGE, dtype=torch.uint8)), (4, CACHE[0]),
                        (6, 16.0), (6, 32)],
    "cache_read_fp4": [(1, SLOTS.int()), (1, SLOTS[:8]), (2, CACHE[:2]), (3, CACHE.view(torch.int8)), (4, 32), (5, KV[:8]), (6, KV.bfloat16()),
                       (5, torch.zeros(9, 4, 64)[:, ::2]), (4, None)],
    "commit_fp4": [(1, CU.long()), (2, I32[:1]), (3, torch.zeros(1, 5, dtype=torch.int32)), (4, KV[:8]), (5, KV.bfloat16()), (6, CACHE[:2]),
                   (7, CACHE[..., 16:]), (8, torch.zeros(1, 3, dtype=torch.int32)), (9, I32.long()), (10, 1.5)],
    "attention_fp4": [(4, CACHE[:2]), (5, CACHE.view(torch.int8)), (4, CACHE[..., :-16]), (12, 32), (12, 1.0)],
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
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            call(*args)
        assert not called, (at, wrong)
    with pytest.raises(TypeError):
        call(*CALLS[name][:-1])


def test_parts_of_a_projection_are_taken_as_they_lie(native):
    module, called, entry = native
    module.prompt(0, FUSED[:, :8], FUSED[:, 8:10], FUSED[:, 10:], CU, 0.1, None, None, False)
    assert called.pop()


def test_tensors_off_the_gpu_are_refused():
    lib = object.__new__(B.SmartTree)
    lib._native, lib._h, lib.device = None, None, 0
    with pytest.raises(ValueError):
        lib.prompt_attention(Q, KV, KV, CU, 0.1)
    with pytest.raises(ValueError):
        lib.kv_cache_write_fp4(KV, KV, SLOTS, CACHE, CACHE, 16)
    with pytest.raises(ValueError):
        lib.kv_cache_read_fp4(SLOTS, CACHE, CACHE, 64, 16)
    with pytest.raises(ValueError):
        lib.tree_commit_fp4(CU, I32, I32, KV, KV, CACHE, CACHE, I32, I32, 16)
    with pytest.raises(ValueError):
        lib.tree_verify_attention(Q, KV, KV, CACHE, CACHE, I32, I32, CU, SLOTS, 0.1, 1, kv_cache_dtype=7)
    with pytest.raises(ValueError):
        lib.tree_verify_attention(Q, KV, KV, CACHE, CACHE, I32, I32, CU, SLOTS, 0.1, 1, kv_cache_dtype=B.SMART_FP4_E2M1)


def test_tensors_on_another_gpu_are_refused():
    lib = object.__new__(B.SmartTree)
    lib._native, lib._h, lib.device = None, None, 0
    there = types.SimpleNamespace(get_device=lambda: 1, device=torch.device("cuda", 1), shape=(9, 8, 64))
    for call in (lambda: lib.prompt_attention(there, KV, KV, CU, 0.1), lambda: lib.kv_cache_write_fp4(there, KV, SLOTS, CACHE, CACHE, 16),
                 lambda: lib.kv_cache_read_fp4(SLOTS, there, CACHE, 64, 16)):
        with pytest.raises(ValueError):
            call()
