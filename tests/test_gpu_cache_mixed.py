"""Prompts and single tokens in one batch behind long prefixes, against the oracle: whether
the prefix is shared, cut or taken by each sequence, the rows get the same.
"""
import pytest

from tests.cache_case import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(28, 4), (4, 4), (8, 2)])
@pytest.mark.parametrize("counts", [[40, 1], [1] * 9 + [150], [1, 60, 0, 2, 1, 33]])
@pytest.mark.parametrize("prefix", [[300], [2500], [6100, 70]])
@pytest.mark.parametrize("layout", ["packed", "padded"])
def test_prompts_beside_tokens(gpu_lib, layout, prefix, counts, heads):
    S = len(counts)
    b = Batch(counts, [n + (13 * s) % 40 for s, n in enumerate(counts)], heads=heads, D=64, page=64, layout=layout,
              prefix=prefix, cuts=[0, S] if len(prefix) == 1 else [0, S // 2, S], seed=S)
    b.upload()
    b.check(*b.attend())
    b.check(*b.attend(see_all=True), see_all=True)
