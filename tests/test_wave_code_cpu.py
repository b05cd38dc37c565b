"""What the source of the kernels has to say by itself where the lanes of a wave work together: a value that comes from another lane is
fetched where that lane is active, and a wave's own exchange through LDS is ordered.  (Neither shows in results while a compiler happens to
keep what it need not.)"""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_22033_amd", "csrc")
CROSS_LANE = re.compile(r"readlane|__shfl|__ballot|dpp_")


def _function(path, name):
    """The text of a function's body, from its name on."""
    text = open(os.path.join(CSRC, path)).read()
    at = re.search(r"\b" + name + r"\([^;{]*\) \{", text)
    depth, i = 1, at.end()
    while depth:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
    return text[at.end():i - 1]


def test_moves_come_from_active_lanes():
    # these are called in a loop that lanes leave at different turns
    for name in ("move_table", "move_tokens"):
        assert not CROSS_LANE.search(_function("sip_beam.h", name)), name
    # and in the kernels nothing is fetched from another lane behind the first loads that some lanes alone make
    for name, first in (("state_reorder_group_kernel", "move_tokens("), ("state_reorder_kernel", "reinterpret_cast<const StateLine*>")):
        body = _function("sip_beam.h", name)
        assert first in body and not CROSS_LANE.search(body[body.index(first):]), name


def test_a_wave_s_counters_are_ordered():
    # Every access of sort_entries() to the wave's counters is one lane's of what another wrote: behind a wave's or the workgroup's barrier since the last.
    body = _function("sip_embed.h", "sort_entries")
    order = re.compile(r"wave_order\(\)|__syncthreads\(\)")
    accesses = [m.start() for m in re.finditer(r"\bat\[w\]\[digit\]", body)]
    assert len(accesses) == 3
    cleared = body.index("at[w][lane] = 0")
    for before, at in zip([cleared] + accesses, accesses):
        assert order.search(body, before, at), body[before:at]
