"""Pointers of asd_rules_verify and asd_rules_logits that are not on their words' boundaries are refused (no GPU needed)."""
import pytest

from paper_2608_03447_gb300 import asd

ALIGN = 6
RULES = asd._RULES.pack(0x1000, 0x2000, 0, 0, 0, 0, 0, 0, 2, 100)


@pytest.mark.parametrize("name", ("draft", "ledger", "a", "c", "rec", "arg", "reg", "status"))
@pytest.mark.parametrize("off", (1, 2))
def test_verify(name, off):
    a = dict(logits=0x4000, draft=0x5000, ledger=0x6000, a=0x7000, c=0x7100, rec=0x7200, arg=0x7300, reg=0x7400,
             status=0x7500, ws=0x10000, wsb=1 << 30, dtype=asd.BF16, K=3, gate=1.0, cap=2)
    a[name] += off
    assert asd.load().asd_rules_verify(RULES, asd._RULES_BLOCK.pack(*a.values()), None) == ALIGN


@pytest.mark.parametrize("off", (1, 2))
def test_logits(off):
    assert asd.load().asd_rules_logits(RULES, 0x4000, asd.F32, 4, 0x5000 + off, 0x8000, None) == ALIGN
