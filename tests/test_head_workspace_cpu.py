"""Workspaces of the vocabulary head: what is enough for a batch is enough for a smaller one.  No GPU: a backward pass that is
asked for no gradient checks its workspace and enqueues nothing."""
import random

import pytest

import paper_2506_22033_amd as sip
from paper_2506_22033_amd import binding, head

COUNTS = [1, 2, 16, 31, 32, 33, 63, 64, 65, 90, 100, 127, 128, 129, 200, 256, 257, 384, 500, 512, 513, 1000, 1024, 2000, 2048, 4096, 5000,
          8192, 20000, 65535, 65536]


def _backward(N, V, D, room):
    return head._load().sip_xent_backward(0x10000, N, D, D, 0x20000, V, D, 0x30000, 1.0, 0x40000, 0x50000, None, 1.0, None, 0, None, 0,
                                          0x100000, room, None)


@pytest.mark.parametrize("V", [1, 300, 4096, 32000, 128256, 151643, sip.SIP_MAX_V])
@pytest.mark.parametrize("D", [8, 64, 512, 1024, 4096, 9272, sip.SIP_MAX_D])
def test_a_workspace_serves_smaller_batches(V, D):
    for backward in (False, True):
        sizes = [sip.sip_xent_workspace_bytes(n, V, D, backward) for n in COUNTS]
        assert sizes == sorted(sizes) and sizes[0] > 0
    for i, n in enumerate(COUNTS):
        room = sip.sip_xent_workspace_bytes(n, V, D, True)
        assert sip.sip_xent_workspace_bytes(n, V, D, False) <= room
        for m in COUNTS[:i + 1]:
            assert _backward(m, V, D, room) == binding.SIP_OK, (n, m)


def test_a_workspace_serves_smaller_batches_of_any_shape():
    rng = random.Random(7)
    for _ in range(3000):
        V, D, N = int(2 ** rng.uniform(0, 19)), 8 * int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 16))
        room, only = sip.sip_xent_workspace_bytes(N, V, D, True), sip.sip_xent_workspace_bytes(N, V, D, False)
        for m in {1, min(N, 64), max(1, N - 1), N, rng.randint(1, N), int(2 ** rng.uniform(0, 16)) % N + 1}:
            assert _backward(m, V, D, room) == binding.SIP_OK, (N, m, V, D)
            assert sip.sip_xent_workspace_bytes(m, V, D, True) <= room and sip.sip_xent_workspace_bytes(m, V, D, False) <= only


def test_the_other_workspaces_grow_with_their_counts():
    for hidden in (32, 2080, 16384):
        for group in (32,):
            sizes = [sip.sip_head_workspace_bytes(n, 1000, hidden, group) for n in range(1, 600)]
            assert sizes == sorted(sizes)
    sizes = [sip.sip_grad_clip_workspace_bytes(n) for n in range(0, 1000)]
    assert sizes == sorted(sizes)
