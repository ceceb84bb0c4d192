"""The 4-bit calls under the checked build: the library tests its indexes, in a process of its own that asks for the outcome at its end."""
import os
import subprocess
import sys

import pytest

from paper_2312_08053_b200 import build as kbuild

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import sys
import pytest
failed = pytest.main(["-x", "-q"] + sys.argv[1:])
from paper_2312_08053_b200 import binding as kb
ctx = kb.new_context([100], 1, [1.0])
assert kb.kimad_debug_check(ctx) == (True, 0, 0), kb.kimad_debug_check(ctx)
assert not failed
print("indexes fine")
"""


def test_messages_operands_and_products():
    if os.environ.get("KIMAD_CHECKED") == "1":
        pytest.skip("this process runs the checked build")
    kbuild.build(checked=True)
    files = [f"tests/test_gpu_mx4{f}.py" for f in ("_product", "_forms", "_layouts", "_pairs", "_parts", "_edges")]
    res = subprocess.run([sys.executable, "-c", CODE] + files, cwd=ROOT, env=dict(os.environ, KIMAD_CHECKED="1"), capture_output=True, text=True, timeout=900)
    assert res.returncode == 0 and "indexes fine" in res.stdout, res.stdout[-3000:] + res.stderr[-2000:]
