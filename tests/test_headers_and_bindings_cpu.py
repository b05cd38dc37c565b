"""Every entry point that a header declares has its signature in the binding, and the other way round."""
import os
import re

import pytest

from paper_2506_22033_amd import beam, head

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")


@pytest.mark.parametrize("header,module", [("sip_beam.h", beam), ("sip_head.h", head)])
def test_the_binding_has_what_the_header_declares(header, module):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, header)).read(), flags=re.S)
    declared = re.findall(r"^(?:size_t|sip_status|int|const char\*)\s+(sip_[a-z_]+)\s*\(([^;]*)\);", text, flags=re.M | re.S)
    assert len(declared) >= 3 and {name for name, _ in declared} == set(module._SIGNATURES)
    for name, arguments in declared:
        assert len(module._SIGNATURES[name][1]) == len(arguments.split(",")), name
