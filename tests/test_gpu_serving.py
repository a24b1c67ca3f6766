"""The example that routes, forks, appends and attends, run as it stands."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def test_serve_instance_example():
    """Every answer's logits are those of the request computed by itself, up to roundings.

    A layer rounds its rows to bfloat16 about eight times (2^-9 each of the row): over two layers both ways of
    computing are within 2 * 8 * 2^-9 = 2^-5 of the exact logits, so within 2^-4 of each other.
    """
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import serve_instance
    finally:
        sys.path.pop(0)
    r = serve_instance.main(say=lambda s: print(s, flush=True))
    assert r["requests"] > 10 and r["matched"] > 0
    assert r["pages"] <= r["before"]
    assert r["worst"] <= 2.0 ** -4
