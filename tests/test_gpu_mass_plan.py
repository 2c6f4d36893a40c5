"""The drawn weight on the GPU in every form that a call may take, with pieces of one chunk and of several, against the definition in 64 bits
(tolerance: mass_cases.Shared.check).  What each case selects is asserted in test_mass_plan."""
import pytest

from mass_cases import CASES, Shared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["random", "stairs"])
@pytest.mark.parametrize("c,dtype", [pytest.param(c, t, id=f"{c['name']}-{t}") for c in CASES for t in c["dtypes"]])
def test_every_form(c, dtype, kind):
    Shared(c, dtype, kind).check()


AT_THE_BOUND = ["few_own", "few_joined", "few_32_own", "few_again", "few_32_again", "many", "many_whole_128", "many_in_turns_frames",
                "many_in_turns_small", "many_in_turns_70"]


@pytest.mark.parametrize("kind", ["high", "low"])
@pytest.mark.parametrize("c,dtype", [pytest.param(c, t, id=f"{c['name']}-{t}") for c in CASES if c["name"] in AT_THE_BOUND for t in c["dtypes"]])
def test_scores_at_the_end_of_their_range(c, dtype, kind):
    """Close to 2^28 and to -2^28, the bound that the header gives; they differ by 16 and 32."""
    Shared(c, dtype, kind).check()
