"""Are the pins of oracle/paged.py strong enough?  Each case plants one plausible mistake in it (oracle_paged_mutants.py) and runs its pins in
a fresh interpreter: they must fail, and pass on the oracle as it is.  CPU only."""
import os
import subprocess
import sys

import pytest

from oracle_paged_mutants import MUTANTS, PIN_FILES

HERE = os.path.dirname(os.path.abspath(__file__))


def run_pins(mutant=None):
    env = dict(os.environ)
    env.pop("SDLLM_ORACLE_MUTANT", None)
    if mutant:
        env["SDLLM_ORACLE_MUTANT"] = mutant
    env["PYTHONPATH"] = HERE + os.pathsep + env.get("PYTHONPATH", "")
    return subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-p", "oracle_paged_mutants", "-m", "not gpu"]
                          + [os.path.join(HERE, f) for f in PIN_FILES], cwd=HERE, env=env, capture_output=True, text=True)


def test_the_oracle_passes_its_pins():
    r = run_pins()
    assert r.returncode == 0, r.stdout[-2000:]


@pytest.mark.parametrize("name", sorted(MUTANTS))
def test_planted_mistake_is_caught(name):
    r = run_pins(name)
    assert r.returncode == 1 and "failed" in r.stdout, f"no pin noticed the mistake '{name}':\n" + r.stdout[-1500:]
