"""prompt_attention refuses what its grid cannot count, before the GPU is asked for anything."""
import pytest

from paper_2604_09731_amd import binding as B
from tests.test_fp4_prompt_arguments import _prompt


@pytest.mark.parametrize("bad", [dict(batch=1 << 23), dict(batch=2 ** 31 - 1, num_kv_heads=8), dict(batch=2 ** 31 - 1, num_kv_heads=1, k_stride=64, v_stride=64),
                                 dict(dtype=B.SMART_F32, batch=1 << 22), dict(dtype=B.SMART_F32, batch=(1 << 23), num_kv_heads=1)])
def test_more_prompts_than_a_grid_holds(bad):
    assert _prompt(**dict(dict(k_stride=512, v_stride=512), **bad)) == B.SMART_EINVAL
