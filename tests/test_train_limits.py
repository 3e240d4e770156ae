"""Limits of include/hmoe_train.h that are refused before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_1704_06363_amd import hmoe


def _join(eps):
    return ctypes.byref(hmoe.Join(64, 1, 1, 1, 1.0, eps, None, None))


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1.17e-38])
def test_norms_refuse_an_eps_whose_inverse_is_infinite(eps):
    lib = hmoe.lib()
    for rc in (lib.hmoe_join_forward(_join(eps), 10, 16, 32, None, 64, 128, None),
               lib.hmoe_join_backward(_join(eps), 10, 16, 32, None, 16, 16, 64, 128, None, None, None, 16, 1 << 40, None)):
        assert rc == -1 and "eps" in hmoe.last_error(), (rc, hmoe.last_error())
    assert lib.hmoe_join_workspace(_join(eps), 10) == 0
    assert lib.hmoe_join_workspace(_join(1.1754944e-38), 10) > 0
