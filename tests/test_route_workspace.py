"""Which calls the one-workgroup form of the router takes, by the work space that they need (no GPU needed)."""
import pytest

from paper_2505_15511_amd import _build, binding


@pytest.fixture(scope="module")
def lib():
    if _build.is_stale():
        _build.build_library()
    return binding.load_library()


def test_one_workgroup_stays_within_64_kb_of_lds(lib):
    """A counter an expert and a word a slot, 16,384 words in all; the other form keeps counts in work space."""
    for n, experts, k in ((1, 1, 1), (1, 256, 2), (100, 50, 2), (1, 16376, 8), (2, 16370, 7), (1024, 32, 8)):
        assert experts + n * k <= 16384 and lib.nomad_route_workspace(n, experts, k) == 0
    for n, experts, k in ((1, 16384, 1), (1, 16377, 8), (2, 16384, 8), (2, 16372, 8)):
        assert experts + n * k > 16384 and lib.nomad_route_workspace(n, experts, k) == 2 * experts * 4   # (one chunk of counts, the totals)


def test_what_is_no_call_needs_none(lib):
    for n, experts, k in ((0, 256, 2), (-1, 256, 2), (5, 0, 1), (5, 16385, 1), (1 << 40, 256, 2)):
        assert lib.nomad_route_workspace(n, experts, k) == 0
