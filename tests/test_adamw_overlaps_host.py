"""AdamW's plan refuses tensors that share memory: the step's blocks would update it at the same time."""
import pytest

from paper_2412_06355_gb300 import binding


def test_parts_that_meet_are_no_overlap():
    binding._refuse_overlaps([(64, 32, "b"), (0, 64, "a"), (96, 0, "empty"), (96, 4, "c"), (80, 0, "empty too")])


@pytest.mark.parametrize("parts", [[(64, 32, "b"), (0, 65, "a")], [(8, 8, "a"), (8, 8, "b")], [(0, 100, "a"), (10, 1, "b")],
                                   [(300, 4, "z"), (200, 101, "y"), (0, 4, "x")]])
def test_overlaps_are_refused_by_name(parts):
    with pytest.raises(ValueError, match="lies in the memory of"):
        binding._refuse_overlaps(parts)
