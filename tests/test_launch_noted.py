"""An attention launch is noted in the launch order when it is in the stream, not when it is tried: what comes
behind a launch that failed may not take the append's rows for waited for."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2609_31224_gb300", "csrc")


@pytest.mark.parametrize("name", ["kvc_prompt.cu", "kvc_weights.cu", "kvc_kv4_attn.cu"])
def test_a_launch_is_noted_once_it_is_made(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    noted = list(re.finditer(r"order->launched(?:_pages)?\(", text))
    assert noted
    for m in noted:
        # In a branch on the launch's result, or behind the return of one that failed.
        before = text[max(0, m.start() - 120):m.start()]
        assert re.search(r"== cudaSuccess\)\s*(\{[^}]*)?$|!= cudaSuccess\) return e;[^}]*$", before), before
