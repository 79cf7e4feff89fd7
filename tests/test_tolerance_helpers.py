"""The tolerance helpers of the GPU tests: what they let pass and what they
reject, results that are not finite among it (no GPU)."""
import numpy as np
import pytest

from vzt import check_close, check_rel

HELPERS = pytest.mark.parametrize("check", [check_close, check_rel])


@HELPERS
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("where", [(slice(None),) * 2, (1, 2), (0, 0)])
def test_a_result_that_is_not_finite_fails(check, bad, where):
    ref = np.arange(1.0, 13.0).reshape(3, 4)
    got = ref.copy()
    got[where] = bad
    with pytest.raises(AssertionError, match="what: element"):
        check(got, ref, 1e-2, "what")


@HELPERS
def test_a_reference_that_is_not_finite_passes_nothing(check):
    for x in (np.nan, np.inf):
        with np.errstate(invalid="ignore"), pytest.raises(AssertionError):
            check(np.full((2, 2), x), np.full((2, 2), x), 1e-2)


@HELPERS
def test_the_allowed_error_and_one_above_it(check):
    ref = np.full((2, 5), -3.0)
    most = 3e-3 if check is check_rel else 6e-3  # rtol |ref|, and rtol times the row's root mean square
    assert check(ref, ref, 1e-3) == 0.0
    assert check(ref + 0.99 * most, ref, 1e-3) == pytest.approx(0.99)
    got = ref.copy()
    got[1, 3] += 1.01 * most
    with pytest.raises(AssertionError, match=r"\(.*1.*3.*\)"):
        check(got, ref, 1e-3)


@HELPERS
def test_shapes_have_to_agree(check):
    assert check(np.zeros((0, 4)), np.zeros((0, 4)), 1e-3) == 0.0
    with pytest.raises(AssertionError):
        check(np.zeros((2, 4)), np.zeros((4, 2)), 1e-3)
