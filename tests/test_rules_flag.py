"""ASD_FLAG_EMPTY_ROWS on the host: asd_rules_verify takes it with either type, and nothing else beside it (no GPU needed)."""
import pytest

from paper_2608_03447_gb300 import asd

DTYPE, OK = 3, 0


@pytest.mark.parametrize("dtype,code", [(asd.F32 | asd.FLAG_EMPTY_ROWS, OK), (asd.BF16 | asd.FLAG_EMPTY_ROWS, OK),
                                        (asd.F16 | asd.FLAG_EMPTY_ROWS, DTYPE), (asd.BF16 | 0x400, DTYPE),
                                        (asd.F32 | asd.FLAG_EMPTY_ROWS | asd.RESIDENT_INPUTS, DTYPE)])
def test_types(dtype, code):
    nothing = asd._RULES.pack(0, 0, 0, 0, 0, 0, 0, 0, 0, 100)  # no requests: nothing is launched
    block = asd._RULES_BLOCK.pack(*[0] * 11, dtype, 3, 1.0, 2)
    lib = asd.load()
    assert lib.asd_rules_verify(nothing, block, None) == code
    if code == OK:  # only verification has the flag
        assert lib.asd_rules_logits(nothing, None, dtype, 4, None, None, None) == DTYPE
