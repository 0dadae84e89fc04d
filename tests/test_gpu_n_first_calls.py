"""Calls whose shared memory is at the most that a kernel has without asking for
more: the sizes around it, each way in a process of its own whose first call
that is, the smallest first."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))

FORK = """
import test_gpu_l_kv_pages as pages
rows, bt = 8192, 16
rng = np.random.RandomState(1)
lens = np.concatenate([rng.randint(1, 40, 4096), np.zeros(4096, int)])
table, shared, free = ref.requests(list(lens), bt, 20000, 2)
pool, cursor = ref.ring(free, 20000, 19990)
for both in (12272, 12273, 12288, 12289):      # rows and pairs
    pairs = both - rows
    dst = np.concatenate([4096 + rng.permutation(4096), [-1]])[:pairs]
    pages.fork(rng.randint(0, 4096, pairs), dst, lens, table, shared, pool, cursor, bt)
"""

COMPACT = """
import test_gpu_l_kv_pages as pages
lens = np.array([700, 0, 33, 1599])
for n in (196096, 196097, 196608, 196609):     # blocks
    table, shared, _ = ref.requests(list(lens), 16, n, n, 2)
    pages.compact(lens, table, shared, 16, in_place=%s)
"""

TABLES = """
import test_gpu_a_kv_tables as tables
rng = np.random.default_rng(3)
for R in (6111, 6112, 6143, 6144):             # requests
    have, fresh = rng.integers(0, 50, R), rng.integers(0, 4, R)
    table, pool, cursor = tables.state(rng, have, fresh, 16)
    _, _, starts, lens, _ = tables.call(have, fresh, table, pool, cursor, 16, int(fresh.sum()))
    assert (starts == np.concatenate([[0], np.cumsum(fresh)])).all() and (lens == have + fresh).all()
    tables.hs.hs_get_device_error()
"""


@pytest.mark.parametrize("code", [FORK, COMPACT % False, COMPACT % True, TABLES],
                         ids=["fork", "compact", "compact_in_place", "tables"])
def test_first_call_of_a_process(code):
    begin = "import sys\nsys.path[:0] = [%r, %r]\nimport numpy as np\nimport pages_testutil as ref\n" % (
        os.path.dirname(HERE), HERE)
    r = subprocess.run([sys.executable, "-c", begin + code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
