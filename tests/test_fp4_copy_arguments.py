"""Copies to and from a 4-bit cache whose grid would not count their threads are refused before the GPU is asked for anything."""
import pytest

from paper_2604_09731_amd import binding as B
from tests.test_fp4_prompt_arguments import _read, _write


@pytest.mark.parametrize("bad", [dict(n=1 << 27), dict(n=2 ** 31 - 1), dict(n=1 << 27, src=B.SMART_F32)])
def test_more_tokens_than_a_grid_holds(bad):
    assert _write(**bad) == B.SMART_EINVAL and _read(**bad) == B.SMART_EINVAL
