"""What importing the package needs (no GPU)."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2504_16068_amd")
TP = os.path.join(PKG, "liballegro_tp.so")

pytestmark = pytest.mark.skipif(not os.path.exists(TP), reason="libraries not built (run __graft_entry__.build())")


def _python(code, path):
    res = subprocess.run([sys.executable, "-c", code], cwd=path, capture_output=True, text=True,
                         env={**os.environ, "PYTHONPATH": str(path)}, timeout=300)
    assert res.returncode == 0, res.stderr
    return res.stdout.strip()


def test_the_package_imports_without_the_latent_library(tmp_path):
    """A tree with liballegro_tp.so alone serves the tensor product; names of the latent track say what is missing."""
    pkg = tmp_path / "paper_2504_16068_amd"
    pkg.mkdir()
    for f in os.listdir(PKG):
        if f.endswith(".py") or f == "liballegro_tp.so":
            os.symlink(os.path.join(PKG, f), pkg / f)
    assert _python("""
import paper_2504_16068_amd as at
assert at.__file__.startswith(%r), at.__file__
plan = at.allegro_tp_plan_create(2, 64)
for use in ("at.allegro_group_rows", "at.ALLEGRO_ACT_SILU"):
    try:
        eval(use)
    except ImportError as e:
        assert "liballegro_latent.so is not built" in str(e), e
    else:
        raise SystemExit("no ImportError")
try:
    from paper_2504_16068_amd import allegro_rms_norm_forward
except ImportError as e:
    pass
else:
    raise SystemExit("no ImportError")
try:
    at.no_such_name
except AttributeError:
    print("ok", plan.d2)
""" % str(tmp_path), tmp_path) == "ok 9"


@pytest.mark.skipif(not os.path.exists(os.path.join(PKG, "liballegro_latent.so")), reason="library not built")
def test_a_whole_tree_has_the_latent_names():
    assert _python("""
from paper_2504_16068_amd import *
import paper_2504_16068_amd as at
assert allegro_group_rows is at.latent.allegro_group_rows and "allegro_rms_norm_fp8" in dir(at)
print("ok", ALLEGRO_ACT_SILU)
""", ROOT) == "ok 1"
