"""What the package gives where the operators behind the decode cannot be had: everything else, and an error when one of them is called."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def python(where, lines):
    return subprocess.run([sys.executable, "-c", lines], cwd=where, env={**os.environ, "PYTHONPATH": str(where)}, capture_output=True, text=True)


@pytest.mark.parametrize("before", ["", "import sys; sys.modules['torch'] = None\n"])
def test_import_star_of_a_tree_that_is_not_built(tmp_path, before):
    held = tmp_path / "paper_1911_00472_amd"
    held.mkdir()
    for f in os.listdir(os.path.join(ROOT, "paper_1911_00472_amd")):
        if f.endswith(".py"):
            shutil.copy(os.path.join(ROOT, "paper_1911_00472_amd", f), held / f)
    p = python(tmp_path, before + "from paper_1911_00472_amd import *\nassert Record and E_RANGE == -5\n"
               "try:\n    rotate_axes(None, None, None, None, None)\nexcept (RuntimeError, ImportError) as e:\n    print('said:', e)")
    assert p.returncode == 0 and "said:" in p.stdout, p.stderr
    p = python(tmp_path, before + "import paper_1911_00472_amd as pcr\ntry:\n    pcr.distill_step(None, None, None, None)\nexcept (RuntimeError, ImportError):\n    print('said')")
    assert p.returncode == 0 and "said" in p.stdout, p.stderr


def test_import_star_of_a_tree_that_is_built():
    p = python(ROOT, "from paper_1911_00472_amd import *\nimport paper_1911_00472_amd.train as train\nassert rotate_axes is train.rotate_axes and distill_loss is train.distill_loss\nprint('had')")
    assert p.returncode == 0 and "had" in p.stdout, p.stderr
