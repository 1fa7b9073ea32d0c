"""The paged 8-bit cache's suites once more under the -DDART_DEBUG build, whose index checks stand in front of its stores (cache
codes, outputs, partial results, tables, page lists): a check that fails skips the store and records an error in the status word,
which these suites assert to be clean."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_suites_of_the_8_bit_cache_are_clean_under_the_debug_build():
    from paper_2601_19278_b200 import build
    env = dict(os.environ, DART_LIB=build.build_debug())
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_kv8.py", "tests/test_gpu_kv8_owned.py", "tests/test_gpu_kv8_padding.py", "-x", "-q",
                        "-m", "gpu", "-p", "no:cacheprovider"], cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-3000:]
