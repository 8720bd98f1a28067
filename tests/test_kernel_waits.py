"""Bounded waits of the kernels whose roles go on as whole warps: a wait's outcome is each lane's own, and
lanes that it sent different ways would not meet again at the next warp-wide instruction.  Looked for in the
source: a run has no way to let a wait give up for some lanes of a warp and not for others."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_37617_gb300", "csrc")


@pytest.mark.parametrize("name", ["k_prompt.cu", "k_attn4_wide.cu"])
def test_outcomes_of_waits_are_agreed_on(name):
    """Nothing goes by one lane's outcome but where one lane alone waits; whole() and __all_sync() take
    them together."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert "auto wait = [&]" in text and re.search(r"\b(whole|__all_sync)\((~0u, )?wait\(", text)
    alone = [line.strip() for line in text.splitlines() if re.search(r"(=|!|&&|\|\||\?|return) *wait\(", line)]
    loads = "if (n >= NST && !wait(&empty[s], (n / NST - 1) & 1)) break;"  # (by one thread)
    assert [line for line in alone if line != loads and "lane == 0 && wait(" not in line] == []
