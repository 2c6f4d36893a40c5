"""The drawn weight on the GPU in every form that a call may take, with pieces of one chunk and of several, against the definition in 64 bits
(tolerance: mass_cases.Shared.check).  What each case selects is asserted in test_mass_plan."""
import pytest

from mass_cases import CASES, Shared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["random", "stairs"])
@pytest.mark.parametrize("c,dtype", [pytest.param(c, t, id=f"{c['name']}-{t}") for c in CASES for t in c["dtypes"]])
def test_every_form(c, dtype, kind):
    Shared(c, dtype, kind).check()
