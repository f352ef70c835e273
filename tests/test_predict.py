"""The prediction library (include/als_predict.h) without a GPU: it builds, exports what its header declares, keeps the
device-code rules, and refuses what it can refuse before touching a device; and the tests' 64-bit forms."""
import ctypes
import os
import re

import numpy as np
import pytest

from tests import predict_oracle
from tests.test_abi import _device_disassembly

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    src = open(os.path.join(ROOT, "include", "als_predict.h")).read()
    return re.sub(r"/\*.*?\*/", "", src, flags=re.S)


def test_library_exports_every_declared_symbol():
    from paper_1603_03820_amd import predict
    declared = set(re.findall(r"\b(als_[a-z_]+)\s*\(", _header()))
    lib = ctypes.CDLL(predict.LIB_PATH)
    assert declared == set(predict.EXPORTED)
    assert not [fn for fn in declared if not hasattr(lib, fn)]


def test_constants_match_the_header():
    from paper_1603_03820_amd import predict
    numbers = dict(re.findall(r"#define (ALS_PREDICT_\w+_MAX) (\d+)", _header()))
    for name in ("ALS_PREDICT_F_MAX", "ALS_PREDICT_N_MAX", "ALS_PREDICT_TOP_MAX"):
        assert int(numbers[name]) == getattr(predict, name)
    acts = {k.lower(): int(v) for k, v in re.findall(r"ALS_ACT_(\w+) = (\d)", _header())}
    assert acts == predict.ACTIVATIONS


def test_header_compiles_as_c():
    import subprocess
    import tempfile
    with tempfile.NamedTemporaryFile("w", suffix=".c") as f:
        f.write('#include "als_predict.h"\nint main(void) { als_scores s; als_given g; (void)s; (void)g; return 0; }\n')
        f.flush()
        subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), f.name],
                       check=True)


def test_structures_match_the_header():
    """The binding's structures have the C compiler's sizes."""
    import subprocess
    import tempfile
    from paper_1603_03820_amd import predict
    with tempfile.TemporaryDirectory() as d:
        src = os.path.join(d, "s.c")
        open(src, "w").write('#include <stdio.h>\n#include <stddef.h>\n#include "als_predict.h"\nint main(void) { printf("%zu %zu %zu %zu",'
                             ' sizeof(als_scores), sizeof(als_given), offsetof(als_scores, rated_ptr), offsetof(als_given, each)); return 0; }\n')
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), src, "-o", os.path.join(d, "s")], check=True)
        sizes = [int(v) for v in subprocess.run([os.path.join(d, "s")], capture_output=True, text=True).stdout.split()]
    assert sizes == [ctypes.sizeof(predict._Scores), ctypes.sizeof(predict._Given), predict._Scores.rated_ptr.offset,
                     predict._Given.each.offset]


def test_device_code_shape():
    """gfx950 code; memory is written only through vector instructions; no packed fp32; matrix instructions of both
    16-bit types."""
    if not os.path.exists("/opt/rocm/llvm/bin/clang-offload-bundler"):
        pytest.skip("ROCm LLVM tools not installed")
    from paper_1603_03820_amd import build
    text = _device_disassembly(build.PREDICT_LIB)
    scalar_writes = re.compile(r"\bs_(?:" + "|".join(["st" + "ore", "atom" + "ic", "dcache_" + "wb"]) + r")")
    assert not scalar_writes.search(text)
    assert not re.search(r"\bv_pk_(?:add|mul|fma)_f32", text)
    assert "v_mfma_f32_16x16x32_bf16" in text and "v_mfma_f32_16x16x32_f16" in text


def test_loads_to_lds():
    """The loads to LDS, which are inline assembly: their wait states, M0 to themselves in their kernels, and no assembly
    that writes a register."""
    if not os.path.exists("/opt/rocm/llvm/bin/clang-offload-bundler"):
        pytest.skip("ROCm LLVM tools not installed")
    from paper_1603_03820_amd import build
    from tests.test_serve import lds_load_violations
    text = _device_disassembly(build.PREDICT_LIB)
    assert lds_load_violations(text) == []
    loading = [k for k in re.split(r"\n(?=[0-9a-f]+ <)", text) if re.search(r"buffer_load_dwordx4 .* lds", k)]
    assert len(loading) == 14       # seven shapes of tiles, two types
    for k in loading:
        assert not re.search(r"gpr_idx|v_movrel|s_movrel|s_sendmsg\b", k)
        uses = [line.split("//")[0].strip() for line in k.splitlines() if re.search(r"\bm0\b", line.split("//")[0])]
        assert uses and all(u.startswith("s_mov_b32 m0,") for u in uses), set(uses)
    for b in re.findall(r"\basm volatile\((.*?)\);", open(build.PREDICT_SRC).read(), flags=re.S):
        outputs = b.split(":")[1] if ":" in b else ""
        assert "=" not in outputs and "+v" not in outputs, b


def test_refusals_without_a_device():
    """Null contexts and a device that does not exist."""
    from paper_1603_03820_amd import predict
    lib, P = predict._lib, ctypes.c_void_p
    assert lib.als_predict_workspace_bytes(-1) == 0
    assert lib.als_predict_workspace_bytes(4096) == 0
    h = P()
    buf = (ctypes.c_char * 4096)()
    base = (ctypes.addressof(buf) + 255) // 256 * 256
    assert lib.als_predict_init(None, 0, P(base), 1 << 40) == -1
    assert lib.als_predict_init(ctypes.byref(h), 0, None, 1 << 40) == -3
    assert lib.als_predict_init(ctypes.byref(h), 0, P(base + 8), 1 << 40) == -4
    assert lib.als_predict_init(ctypes.byref(h), 4096, P(base), 1 << 40) == -7
    assert not h.value
    assert lib.als_predict(None, None, 0, 1, None, 0, None, 0, 1, 0, 1, None, None, 0, 0.0, 0.0, None, 0, None, 0, 0,
                           None) == -1
    s, g = predict._Scores(), predict._Given()
    assert lib.als_log_prob(None, ctypes.byref(s), ctypes.byref(g), None, None, None, 0, None, None, None) == -1
    assert lib.als_log_prob_grad(None, ctypes.byref(s), ctypes.byref(g), None, None, None, None, None, None, 0, None,
                                 None) == -1
    assert lib.als_predict_destroy(None) == 0 and lib.als_predict_last_hip_error(None) == 0


def test_training_and_serving_do_without_the_library(tmp_path):
    """The package where libals_predict.so is not built: the rest imports, and the prediction names say what is missing."""
    import shutil
    from tests.test_import import PACKAGE, run
    shutil.copytree(os.path.join(ROOT, PACKAGE), tmp_path / PACKAGE,
                    ignore=shutil.ignore_patterns("libals_predict.so", "__pycache__", "csrc"))
    r = run(tmp_path, f"import {PACKAGE} as p; from {PACKAGE} import driver, serve, recommend; print(p.als_score.__name__)")
    assert r.returncode == 0 and r.stdout.split() == ["als_score"], r.stderr
    for code in (f"from {PACKAGE} import predict", f"from {PACKAGE} import Predictor", f"import {PACKAGE}; {PACKAGE}.als_log_prob"):
        r = run(tmp_path, code)
        assert r.returncode != 0 and "libals_predict.so is not built" in r.stderr, r.stderr


def test_the_names_are_the_packages():
    import paper_1603_03820_amd as p
    from paper_1603_03820_amd import predict
    for name in ("Predictor", "als_predict", "als_log_prob", "als_log_prob_grad", "als_predict_workspace_bytes"):
        assert getattr(p, name) is getattr(predict, name) and name in dir(p)


def test_oracle_by_hand():
    row = predict_oracle.Row(np.log([0.5, 0.25, 0.125, 0.125]))
    assert np.allclose(np.exp(row.log_p), [0.5, 0.25, 0.125, 0.125])
    assert row.entropy == pytest.approx(1.75 * np.log(2))
    assert list(row.top(5)[0]) == [0, 1, 2, 3, -1] and row.top(5)[1][4] == -np.inf
    row = predict_oracle.Row(np.array([1.0, np.nan, 3.0, 3.0, -np.inf]), temperature=0.0)
    assert list(row.top(4)[0]) == [2, 3, 0, -1] and row.log(2) == 0 and row.log(3) == -np.inf and row.entropy == 0
    row = predict_oracle.Row(np.array([np.inf, 1.0, np.inf]))
    assert np.allclose(np.exp(row.log_p), [0.5, 0.0, 0.5]) and row.entropy == pytest.approx(np.log(2))
    row = predict_oracle.Row(np.array([5.0, 1.0]), rated=[0, 1, 7])
    assert row.log(0) == -np.inf and row.entropy == 0 and list(row.top(2)[0]) == [-1, -1]
    y = np.array([-np.inf, -30.0, -1.0, 0.0, 2.0])
    assert np.allclose(predict_oracle.activate(y, "gelu"), [0, 0, -0.15865525, 0, 1.95449974])
    assert np.allclose(predict_oracle.activate(y, "silu"), [0, -30 * np.exp(-30), -0.26894142, 0, 1.76159416])
    out, size = predict_oracle.predict([[1.0, -2.0]], [[3.0, 1.0], [0.0, 1.0]], users=[0, 1], item_offset=[1.0, -1.0],
                                       activation="relu", residual=np.full((2, 2), 0.5))
    assert np.array_equal(out[0], [2.5, 0.5]) and np.isnan(out[1]).all() and np.array_equal(size[0], [6.0, 3.0])


@pytest.mark.parametrize("seed", range(6))
def test_oracle_gradient_against_differences(seed):
    """The formula's gradient against central differences of the loss, with repeated, left-out and far given columns."""
    rng = np.random.default_rng(seed)
    n = 9
    z, t, h = rng.standard_normal(n), 0.4 + rng.random(), rng.standard_normal()
    rated, given = [2, 11], [0, 4, 4, 2, 8, 15, -1]
    g = rng.standard_normal(len(given))
    grad, _ = predict_oracle.Row(z, t, rated).gradient(given, g, h)
    step = 1e-6
    for j in range(n):
        up, down = z.copy(), z.copy()
        up[j] += step
        down[j] -= step
        slope = (predict_oracle.Row(up, t, rated).loss(given, g, h) - predict_oracle.Row(down, t, rated).loss(given, g, h)) / (2 * step)
        assert grad[j] == pytest.approx(slope, abs=1e-7)
    assert grad[2] == 0
