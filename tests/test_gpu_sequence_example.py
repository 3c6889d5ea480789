"""The sequence operators together, as the example trains and serves them."""
import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_sequence_layer_example(built_lib):
    """The loss falls; columns served one by one give the whole line's logits (fp32 sums in another order: 1e-5); the
    8-bit output's logits are within e4m3's half step, 2^-4, of them."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("sequence_layer", os.path.join(ROOT, "examples", "sequence_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    losses, err, err8 = mod.main(steps=25, examples=16)
    print(losses[0], losses[-1], err, err8)
    assert losses[-1] < 0.7 * losses[0]
    assert err < 1e-5
    assert 0 < err8 < 2.0 ** -4
