"""Log probabilities of rows cut in every way that the number of rows can ask
for: chunks of 1, 2, 4 and 8 vectors a thread with a join (1, 2: few rows), and
a block a row (1024 rows and more), with and without alternatives, in every
type. Tolerances as in test_ops_logits.py."""
import pytest
import torch

from test_ops_logits import TYPES, check, logits, some_tokens


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [10, 30, 60, 110, 300, 1100])
def test_every_cut(n, kind):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    x, t = logits(gen, n, 40_003, kind, 2), some_tokens(gen, n, 40_003)
    for top in (0, 6):
        check(x, t, top)
    x[::3, 7:40_000] = -torch.inf          # masked but for a few at both ends
    for top in (0, 6):
        check(x, t, top)
