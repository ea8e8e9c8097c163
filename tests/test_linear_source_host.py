"""What the compiler has to be told about the dense layers' written-out loads (no GPU)."""
import os
import re

import paper_2003_10735_amd as st


def test_loads_into_lds_take_m0_as_an_operand():
    """A statement that set M0 by itself would do so behind the compiler's back, which cannot be told of it by a clobber (the register is reserved)."""
    with open(os.path.join(os.path.dirname(st.__file__), "csrc", "k_linear.hip")) as f:
        statements = re.findall(r"\basm volatile\((.*?)\);", f.read(), re.S)
    loads = [s for s in statements if re.search(r"\blds\b", s)]
    assert loads and all('"{m0}"(' in s for s in loads)
    assert not any(re.search(r"\bm0\b", s.split("::")[0].rsplit('"', 1)[0]) for s in statements)
