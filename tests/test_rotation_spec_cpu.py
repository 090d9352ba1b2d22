"""What a rotation's spec points to stays alive and in place: its tensors cannot be exchanged under the view that the kernels read."""
import pytest

from paper_2203_15952_amd import binding as B


@pytest.mark.parametrize("name", ["gamma_q", "gamma_k", "turns"])
def test_tensors_are_not_exchanged(name):
    spec = B.QkNormRotate.__new__(B.QkNormRotate)
    with pytest.raises(AttributeError):
        setattr(spec, name, None)
