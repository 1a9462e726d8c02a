"""The smoke run reaches every kernel of the paged cache."""
import pytest

import __graft_entry__ as entry
from tests.gpu_util import launches

pytestmark = pytest.mark.gpu


def test_step_reaches_every_kernel(cuda_device):
    _, calls = entry.paged_step()
    for call in calls:  # (functions are set up at their first call, outside of a capture)
        call()
    got = [k[0][0] for k in map(launches, calls)]
    assert got == ["paged_slots_kernel", "qk_norm_rope_kernel", "paged_few_kernel", "paged_few_kernel", "paged_many_kernel"]
    entry.smoke_paged()
