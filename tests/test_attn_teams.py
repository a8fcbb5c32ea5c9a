"""Room for the sums that the CTAs of a team send one another in the kernel for few rows, as its source has it. CPU only."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2206_08869_b200", "csrc")


def _source():
    with open(os.path.join(CSRC, "attn_split.cu")) as f:
        return f.read()


def _places(text, big):
    """Sums of a row that lie between kSums and kKept in either shape."""
    n = re.search(r"kKept = kSums \+ (\w+) \* kCols \* 8", text).group(1)
    if n == "kSumPlaces":
        n = re.search(r"kSumPlaces = kBig \? (\w+) : (\w+);", text).group(1 if big else 2)
        n = re.search(r"\b%s = (\d+)" % n, text).group(1)
    return int(n)


@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("big,teams", [(True, range(2, 17)), (False, (2, 4, 8))])
def test_no_sum_is_written_behind_the_room_for_sums(dim, big, teams):
    """A member writes the sums of dimension d to place member * own + d % own of CTA d / own."""
    text = _source()
    assert "(u.member * own + key % own) * kCols * 8" in text and "(m * own + dl) * kCols + e" in text
    room = _places(text, big)
    for team in teams:
        own = -(-dim // team)
        written = {(d // own, m * own + d % own) for m in range(team) for d in range(dim)}
        assert len(written) == team * dim and max(cta for cta, _ in written) < team
        assert max(place for _, place in written) < room, (team, dim)
