"""The attention of several queries on the GPU, against the definitions in 64 bits."""
import pytest

from tests import cache_cases as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bench(lib):
    return C.Bench(lib, lib.Sttm(0), "cuda:0")


from tests.query_tests import *  # noqa: E402,F401,F403  -- the tests that run on host threads too
from tests.residual_tests import *  # noqa: E402,F401,F403
