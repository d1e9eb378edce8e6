"""The amortised calibration example: its operators run together, training through the
replay's gradients lowers the loss, and streaming agrees with reading at once."""
import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_amortised_fit():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("amortised_fit", os.path.join(ROOT, "examples", "amortised_fit.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    history, apart = m.main(n=4, T=120, steps=25, report=lambda *a, **k: None)
    assert history[-1] < history[0]
    assert apart < 1e-4
