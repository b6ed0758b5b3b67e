"""What the workers' matrix update refuses, on the host: everything that one of its two calls would refuse comes back before the first of them."""
import numpy as np
import pytest

from paper_2009_14783_amd import binding as hs
from paper_2009_14783_amd.step import MatrixUpdate

ADAM = dict(lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8)


@pytest.mark.parametrize("compute", [0, 1])
def test_what_can_be_updated_is_fine(compute):
    o = MatrixUpdate.check(dict(momentum=0.9), ADAM, 8.0, compute)
    assert o == dict(MatrixUpdate.DEFAULTS, momentum=0.9, lr=1e-4)
    MatrixUpdate.check(dict(coeff=np.ones((3, 3)), steps=3), dict(ADAM, weight_decay=0.1), 0.0, compute)
    assert MatrixUpdate.check({}, dict(ADAM, beta1=0.0, beta2=0.0, eps=0.0), 1, compute)["rms"] == 0.2


@pytest.mark.parametrize("adam", [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=float("nan"))])
def test_values_of_adam(adam):
    with pytest.raises(hs.HsError) as e:
        MatrixUpdate.check({}, dict(ADAM, **adam), 8.0, 1)
    assert e.value.status == 1


@pytest.mark.parametrize("missing", ["lr", "beta1", "beta2", "eps"])
def test_values_of_adam_that_are_missing(missing):
    adam = {k: v for k, v in ADAM.items() if k != missing}
    with pytest.raises(KeyError, match=missing):
        MatrixUpdate.check({}, adam, 8.0, 1)
    with pytest.raises(KeyError, match=missing):
        MatrixUpdate.check(dict(lr=1e-3), adam, 8.0, 1)      # the matrices' own rate does not stand in for Adam's


@pytest.mark.parametrize("muon", [dict(steps=70), dict(steps=0), dict(coeff=np.zeros((4, 3))), dict(coeff=np.full((5, 3), np.inf)), dict(momentum=1.0), dict(lr=float("nan")),
                                  dict(weight_decay=float("inf")), dict(rms=-1.0), dict(eps=-1.0)])
def test_values_of_the_matrix_update(muon):
    with pytest.raises(hs.HsError) as e:
        MatrixUpdate.check(muon, ADAM, 8.0, 1)
    assert e.value.status == 1


def test_names_and_weights():
    with pytest.raises(TypeError, match="momentun"):
        MatrixUpdate.check(dict(momentun=0.9), ADAM, 8.0, 1)
    for denom in (-1.0, float("nan"), float("inf")):
        with pytest.raises(hs.HsError):
            MatrixUpdate.check({}, ADAM, denom, 1)
    with pytest.raises((TypeError, ValueError)):
        MatrixUpdate.check({}, dict(ADAM, beta1="0.9x"), 8.0, 1)
