"""examples/event_attention.py: the sequence operators with the event convolution, trained
and then run event by event."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "event_attention.py")


def test_trains_and_runs_event_by_event():
    spec = importlib.util.spec_from_file_location("event_attention", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, worst = m.main(events=1500, steps=25, log=lambda s: print(s, flush=True))
    assert losses[-1] < 0.6 * losses[0]
    # the same float32 products in another order: some hundred roundings of 2^-24
    assert worst < 2.0 ** -16
