"""More of blocks that several rows hold, on the GPU: the largest workers' tables."""
import pytest

from tests import test_kv_pages_gpu as pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [(1, 1024, 16, 262144, 64, 4000, 900), (1, 700, 16, 262144, 40, 70000, 600), (2, 513, 32, 262143, 20, 3, 500)], ids=str)
def test_many_rows_of_the_largest_workers(case):
    """More than two rows to a thread beside as many blocks as a worker may have, with the token list in the step's own launch and in one behind it."""
    pages.test_tables(case)
