"""AdamW's plan refuses tensors that share memory: the step's blocks would update it at the same time."""
import pytest

from paper_2412_06355_gb300 import binding


def test_parts_that_meet_are_no_overlap():
    binding._refuse_overlaps([(64, 32, "m", 1), (0, 64, "param", 0), (96, 0, "v", 2), (96, 4, "copy", 3), (80, 0, "m", 4)])


@pytest.mark.parametrize("parts,message", [
    ([(64, 32, "m", 1), (0, 65, "param", 0)], "m of tensor 1 lies in the memory of param of tensor 0"),
    ([(8, 8, "m", 0), (8, 8, "v", 0)], "v of tensor 0 lies in the memory of m of tensor 0"),
    ([(0, 100, "param", 0), (10, 1, "copy", 5)], "copy of tensor 5"),
    ([(300, 4, "scales", 2), (200, 101, "v", 1), (0, 4, "m", 0)], "scales of tensor 2 lies in the memory of v of tensor 1")])
def test_overlaps_are_refused_by_name(parts, message):
    with pytest.raises(ValueError, match=message):
        binding._refuse_overlaps(parts)
