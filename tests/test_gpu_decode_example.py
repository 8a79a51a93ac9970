"""The example that runs the pruning path and the key-value cache together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_pruned.py")


@pytest.mark.parametrize("argv", [["--requests", "3", "--visual", "200", "--steps", "20"],
                                  ["--requests", "1", "--visual", "33", "--layers", "3", "--steps", "3", "--page", "24"]])
def test_prune_and_decode(argv):
    spec = importlib.util.spec_from_file_location("decode_pruned", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.main([*argv, "--check"])
    n, steps = int(argv[3]), int(argv[argv.index("--steps") + 1])
    for before, after in zip(got["prompt_tokens"], got["cached_after_pruning"]):
        assert after == before - n + -(-n // 8)
    assert got["cached_at_the_end"][:-1] == [c + steps for c in got["cached_after_pruning"]]
    # one rounding to bf16 (2^-8 an element) and what fp32 sums add to it
    assert 0.0 < got["worst_relative_error"] < 2.0 ** -8
