"""The package where only a part of its libraries is built."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = "paper_1603_03820_amd"


def run(where, code):
    return subprocess.run([sys.executable, "-c", code], cwd=where, capture_output=True, text=True, timeout=300)


@pytest.fixture
def copy(tmp_path):
    """The package without libals_serve.so."""
    shutil.copytree(os.path.join(ROOT, PACKAGE), tmp_path / PACKAGE,
                    ignore=shutil.ignore_patterns("libals_serve.so", "__pycache__", "csrc"))
    return tmp_path


def test_training_does_without_the_serving_library(copy):
    r = run(copy, f"import {PACKAGE} as p; from {PACKAGE} import als, driver; print(p.ALS_F_MAX, p.als_half_sweep.__name__)")
    assert r.returncode == 0, r.stderr
    assert r.stdout.split() == ["128", "als_half_sweep"]


def test_the_serving_names_say_what_is_missing(copy):
    for code in (f"from {PACKAGE} import serve", f"from {PACKAGE} import Recommender", f"import {PACKAGE}; {PACKAGE}.als_score"):
        r = run(copy, code)
        assert r.returncode != 0 and "libals_serve.so is not built" in r.stderr, r.stderr
    r = run(copy, f"import {PACKAGE}; {PACKAGE}.no_such_name")
    assert r.returncode != 0 and "AttributeError" in r.stderr


def test_the_serving_names_are_the_packages():
    import paper_1603_03820_amd as p
    from paper_1603_03820_amd import serve
    for name in ("Recommender", "als_quantize", "als_sample", "als_score", "als_serve_workspace_bytes"):
        assert getattr(p, name) is getattr(serve, name) and name in dir(p)
