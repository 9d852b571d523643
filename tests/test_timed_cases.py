"""The timed cases of perf/operators.py that a host can check: the library takes the
layers that they make."""
import importlib.util
import os
import random

import pytest


@pytest.fixture(scope="module")
def cases():
    path = os.path.join(os.path.dirname(__file__), "..", "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("timed_operators", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _create(c, B, N):
    from paper_2606_15615_amd import _lib
    p = _lib.moeca_policy_default()
    p.mode = _lib.MOECA_MODE_THRESHOLD if c["kind"] == "cycle" else _lib.MOECA_MODE_FULL
    p.act = ["gelu_tanh", "gelu_erf", "swiglu"].index(c["act"])
    p.batch, p.tokens, p.n_shared = B, N, c["n_shared"]
    _lib.moeca_layer_destroy(_lib.moeca_layer_create(c["d"], c["E"], c["k"], c["d_ff"], p))


def test_layers_are_taken(cases):
    """Listed ones, the first drawn ones, and draws of more than 32768 branches a sample
    where k does not divide 1024, which go in parts."""
    drawn = [cases.draw(random.Random(s)) for s in list(range(400)) + [5303]]
    odd = dict(cases.draw(random.Random(5303)), N=10937)   # a prime number of tokens
    split = 0
    for c in cases.listed() + drawn + [odd]:
        if c["kind"] not in ("experts", "cycle"):
            continue
        B, N = cases._samples(c)
        assert B * N == c["B"] * c["N"]
        split += N != c["N"]
        _create(c, B, N)
    assert split == 2
