"""The example that runs the reshard and the actor's update together."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_actor_update_improves_its_objective():
    spec = importlib.util.spec_from_file_location("actor_update", os.path.join(ROOT, "examples", "actor_update.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    history = m.main(prompts=8, epochs=4, verbose=False)
    # before the first step every ratio is 1, so the objective is the mean advantage; the clipped objective rises from there
    objectives = [o for o, _ in history]
    assert objectives[1] > objectives[0] and objectives[3] > objectives[0]
    assert all(0 < e < 10.4 for _, e in history)                               # entropies lie below log(32000)
