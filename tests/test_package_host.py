"""The package's face: what it says of itself and what a star import brings."""
import paper_2309_15812_amd


def test_docstring_and_star_import():
    assert "oriented 1D kernels" in paper_2309_15812_amd.__doc__
    names = {}
    exec("from paper_2309_15812_amd import *", names)
    assert {"ops", "block", "synth", "build"} <= set(names)
    assert callable(names["ops"].fwd) and callable(names["build"].build) and names["block"].OrientedBlock
