"""Biases of two to five queries, both sides of where rows are taken in tiles, and of single queries behind long caches: rows of
more pieces than a block has threads."""
import pytest
from test_bias import MAPS, test_bias as compare

pytestmark = pytest.mark.gpu

# batch, heads, queries, keys
SIZES = [(2, 3, 2, 1), (2, 3, 3, 7), (2, 3, 4, 8), (2, 3, 5, 7), (3, 2, 2, 300), (2, 3, 4, 2051), (2, 2, 3, 4097), (3, 2, 5, 4097),
         (2, 2, 1, 4097), (5, 3, 1, 2048), (1, 2, 2, 9000)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("how", MAPS)
def test_bias_of_few_queries(how, size):
    compare(how, size)
