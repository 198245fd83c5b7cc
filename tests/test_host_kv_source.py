"""What the compiler cannot check in the attention's source."""
import os
import re

import paper_2609_02652_amd as P

SOURCE = os.path.join(os.path.dirname(P.__file__), "csrc", "attend.hip")


def test_no_instruction_in_inline_assembly():
    """A matrix product's result may be read only some cycles after it.  The compiler
    counts them for its own instructions, not for those in inline assembly; an empty
    template (which only hides a copy from it) issues none."""
    with open(SOURCE) as f:
        templates = re.findall(r'\basm\b(?:\s+volatile)?\s*\(\s*"([^"]*)"', f.read())
    assert templates and all(t == "" for t in templates), templates
