"""The serving library (include/als_serve.h) without a GPU: it builds, exports what its header declares, keeps the
device-code rules, and refuses what it can refuse before touching a device; and the tests' 64-bit draw."""
import ctypes
import os
import re

import numpy as np
import pytest

from tests.serve_oracle import Draw
from tests.test_abi import _device_disassembly

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    src = open(os.path.join(ROOT, "include", "als_serve.h")).read()
    return re.sub(r"/\*.*?\*/", "", src, flags=re.S)


def test_library_exports_every_declared_symbol():
    from paper_1603_03820_amd import serve
    declared = set(re.findall(r"\b(als_[a-z_]+)\s*\(", _header()))
    lib = ctypes.CDLL(serve.LIB_PATH)
    assert declared == set(serve.EXPORTED)
    assert not [fn for fn in declared if not hasattr(lib, fn)]


def test_limits_match_the_header():
    from paper_1603_03820_amd import serve
    numbers = dict(re.findall(r"#define (ALS_SERVE_\w+_MAX) (\d+)", _header()))
    assert int(numbers["ALS_SERVE_F_MAX"]) == serve.ALS_SERVE_F_MAX
    assert int(numbers["ALS_SERVE_N_MAX"]) == serve.ALS_SERVE_N_MAX
    assert 128 * 128 * serve.ALS_SERVE_F_MAX < 2 ** 31       # the sums of als_score
    assert 2 ** 40 * serve.ALS_SERVE_N_MAX <= 2 ** 62        # the sums of als_sample


def test_device_code_shape():
    """gfx950 code; memory is written only through vector instructions; no packed fp32; integer matrix
    instructions."""
    if not os.path.exists("/opt/rocm/llvm/bin/clang-offload-bundler"):
        pytest.skip("ROCm LLVM tools not installed")
    from paper_1603_03820_amd import build
    text = _device_disassembly(build.SERVE_LIB)
    scalar_writes = re.compile(r"\bs_(?:" + "|".join(["st" + "ore", "atom" + "ic", "dcache_" + "wb"]) + r")")
    assert not scalar_writes.search(text)
    assert not re.search(r"\bv_pk_(?:add|mul|fma)_f32", text)
    assert re.search(r"v_mfma_i32_\w+_i8", text)


def _sgprs(token):
    m = re.match(r"s\[(\d+):(\d+)\]$", token) or re.match(r"s(\d+)()$", token)
    return set(range(int(m.group(1)), int(m.group(2) or m.group(1)) + 1)) if m else set()


def lds_load_violations(text):
    """Loads to LDS (which are inline assembly, so the compiler keeps no wait states for them) that read a scalar
    register less than five wait states after a vector instruction wrote it, or M0 less than one after its write."""
    bad, hist = [], []
    for line in text.splitlines():
        t = line.split("//")[0].strip()
        if t.endswith(">:"):
            hist = []
            continue
        if not t or t.endswith(":"):
            continue
        op = t.split()[0]
        args = [a.strip().split()[0] for a in t[len(op):].split(",") if a.strip()]
        if op == "s_nop":
            hist.append((op, set(), int(args[0], 0) + 1))
            continue
        if op.startswith("buffer_load") and t.split()[-1] == "lds":
            reads = set().union(*(_sgprs(a) for a in args))
            states = 0
            for prior, written, n in reversed(hist):
                if (states < 5 and prior.startswith("v_") and written & reads) or (states < 1 and "m0" in written):
                    bad.append(t)
                    break
                states += n
        written = set()
        if args and op.startswith(("v_", "s_")):
            written = {"m0"} if args[0] == "m0" else _sgprs(args[0])
            if op.startswith("v_cmp") or op.startswith("v_add_co") or len(args) > 1 and op.startswith("v_div_scale"):
                written |= _sgprs(args[min(1, len(args) - 1)])
        hist = (hist + [(op, written, 1)])[-8:]
    return bad


def test_loads_to_lds_settled():
    """The wait states of the loads to LDS, and that the check catches planted violations."""
    if not os.path.exists("/opt/rocm/llvm/bin/clang-offload-bundler"):
        pytest.skip("ROCm LLVM tools not installed")
    from paper_1603_03820_amd import build
    planted = ("<k>:\n\tv_readfirstlane_b32 s9, v1\n\ts_mov_b32 m0, s4\n\ts_nop {}\n"
               "\tbuffer_load_dwordx4 v0, s[8:11], s3 offen lds\n")
    assert len(lds_load_violations(planted.format(2))) == 1
    assert lds_load_violations(planted.format(3)) == []
    assert len(lds_load_violations(planted.replace("s9", "s3").format(0))) == 1
    assert len(lds_load_violations("<k>:\n\ts_mov_b32 m0, s4\n\tbuffer_load_dwordx4 v0, s[8:11], s3 offen lds\n")) == 1
    text = _device_disassembly(build.SERVE_LIB)
    assert len(re.findall(r"buffer_load_dwordx4 .* lds", text)) > 50
    assert lds_load_violations(text) == []


def test_loads_to_lds_have_m0_to_themselves():
    """Kernels with loads to LDS use M0 for nothing else (the compiler does not know that they write it)."""
    if not os.path.exists("/opt/rocm/llvm/bin/clang-offload-bundler"):
        pytest.skip("ROCm LLVM tools not installed")
    from paper_1603_03820_amd import build
    kernels = re.split(r"\n(?=[0-9a-f]+ <)", _device_disassembly(build.SERVE_LIB))
    loading = [k for k in kernels if re.search(r"buffer_load_dwordx4 .* lds", k)]
    assert len(loading) == 18       # six shapes of tiles, three types
    for k in loading:
        assert not re.search(r"gpr_idx|v_movrel|s_movrel|s_sendmsg\b", k)
        uses = [line.split("//")[0].strip() for line in k.splitlines() if re.search(r"\bm0\b", line.split("//")[0])]
        assert uses and all(u.startswith("s_mov_b32 m0,") for u in uses), set(uses)


def test_inline_assembly_has_no_result_in_flight():
    """The library's inline assembly writes no register (loads go to LDS), so nothing can be overwritten by a
    load on its way."""
    source = open(os.path.join(ROOT, "paper_1603_03820_amd", "csrc", "serve.hip")).read()
    blocks = re.findall(r"\basm volatile\((.*?)\);", source, flags=re.S)
    assert blocks
    for b in blocks:
        outputs = b.split(":")[1] if ":" in b else ""
        assert "=" not in outputs and "+v" not in outputs, b


def test_refusals_without_a_device():
    """Null contexts and a device that does not exist."""
    from paper_1603_03820_amd import serve
    lib, P = serve._lib, ctypes.c_void_p
    assert lib.als_serve_workspace_bytes(-1) == 0
    assert lib.als_serve_workspace_bytes(4096) == 0
    h = P()
    buf = (ctypes.c_char * 4096)()
    base = (ctypes.addressof(buf) + 255) // 256 * 256
    assert lib.als_serve_init(None, 0, P(base), 1 << 40) == -1
    assert lib.als_serve_init(ctypes.byref(h), 0, None, 1 << 40) == -3
    assert lib.als_serve_init(ctypes.byref(h), 0, P(base + 8), 1 << 40) == -4
    assert lib.als_serve_init(ctypes.byref(h), 4096, P(base), 1 << 40) == -7
    assert not h.value
    assert lib.als_quantize(None, None, 0, 0, 1, None, 0, 1, None, 1, None, None) == -1
    assert lib.als_score(None, None, 1, None, 0, None, 1, None, 0, 1, None, 0, 1, None) == -1
    assert lib.als_sample(None, None, 0, 0, 0, 0, None, None, None, None, None, 0, None, None, None) == -1
    assert lib.als_serve_destroy(None) == 0 and lib.als_serve_last_hip_error(None) == 0


def test_oracle_draw_by_hand():
    """Four equal columns split the uniform number's range in four; the cuts; the empty row; and a wrong column or
    probability is not accepted."""
    z = np.zeros(4)
    for i in range(4):
        d = Draw(z, (i + 0.5) / 4)
        assert [d.accepts(c, np.log(0.25)) for c in range(4)] == [c == i for c in range(4)]
        assert not d.accepts(i, np.log(0.3))
    assert Draw(z, 0.9, top_k=2).accepts(1, np.log(0.5))
    assert Draw(z, 0.9, top_p=0.6).accepts(2, np.log(1 / 3))
    assert Draw(z, 0.9, rated=[3, 2, 9]).accepts(1, np.log(0.5))
    z = np.log([0.5, 0.25, 0.125, 0.125])
    assert Draw(z, 0.7, min_p=0.4).accepts(1, np.log(1 / 3))
    assert not Draw(z, 0.7, min_p=0.4).accepts(2, np.log(1 / 3))
    assert Draw(z, 0.49).accepts(0, np.log(0.5)) and not Draw(z, 0.51).accepts(0, np.log(0.5))
    assert Draw(z[::-1].copy(), 0.99, temperature=0.0).accepts(3, 0.0)
    assert Draw(np.full(3, -np.inf), 0.5).accepts(-1, -np.inf)
    assert Draw(np.array([1.0, np.nan]), 0.5, rated=[0]).accepts(-1, -np.inf)
