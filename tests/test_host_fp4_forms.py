"""Which form of the products in 4 bits the library launches for the sizes of fp4_forms.py, on a runtime that runs nothing (fake_hip.cpp)."""
import ctypes
import json
import os
import re
import shutil
import subprocess
import sys

import pytest

import fake_hip
import fp4_forms as forms

HERE = os.path.dirname(os.path.abspath(__file__))
A = 0x7000000000                                                 # an address that is never used
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"),
                                reason="needs g++ and the HIP headers")


def _up(n, to):
    return -(-n // to) * to


def _form(name):
    """Of a kernel's name: its tile, or the tiles of 16 that a workgroup of the form for few rows has."""
    size = [int(v) for v in re.findall(r"Li(\d+)E", name)]
    cols = "cols " if "ILb1E" in name else ""
    if "k_fp4_product_thin" in name:
        return "thin %d %d" % tuple(size[:2])
    if "k_fp4_product64" in name:
        return cols + "64x64"
    assert "k_fp4_product" in name, name
    return cols + "%dx%d" % tuple(size[:2])


def _calls():
    """{key: (entry point, arguments)}"""
    out = {}

    def product(key, m, n, k, groups, ld=None, y_type=1, scales=16):
        ld, ls = ld or _up(-(-k // 2), 16), _up(-(-k // 32), scales)
        out[key] = ("tuna_fp4_matmul", [A, ld, A, ls, A, _up(-(-k // 2), 16), n * _up(-(-k // 2), 16), A, ls, n * ls, A if groups > 1 else None, groups, A, y_type, n, m, n, k])

    for form, s in forms.SIZES.items():
        for t in (0, 1):
            product("%s of %d" % (form, t), **s, y_type=t)
    for form in forms.LARGE[:2]:
        for k in forms.LENGTHS:
            product("%s of length %d" % (form, k), **dict(forms.SIZES[form], k=k))
    for i, (form, bounds) in enumerate(forms.RAGGED):
        product("%s ragged %d" % (form, i), bounds[-1] + (2 if bounds[0] else 0), forms.SIZES[form]["n"], 1111, len(bounds) - 1)
    for form, (m, bounds, _) in forms.BOUNDS.items():
        product("%s bounds" % form, m, forms.SIZES[form]["n"], 1100, len(bounds) - 1)
    for form, s in forms.FAR_WEIGHTS.items():
        product("%s far weights" % form, **s)
    for form, ld in forms.FAR_ROWS.items():
        product("%s far rows" % form, **forms.SIZES[form], ld=ld)
    for i, (form, n, k, split) in enumerate(forms.GRADIENT):
        m, groups = split[-1], len(split) - 1
        nb = -(-m // 128) + groups - 1
        out["%s gradient %d" % (form, i)] = ("tuna_fp4_matmul_grad_w", [A, 64 * nb, A, _up(4 * nb, 16), A, 64 * nb, A, _up(4 * nb, 16), A if groups > 1 else None, groups,
                                                                        A, 0, k + 2, n * (k + 2), m, n, k])
    # rows of scales, or a group's, that do not start on 16 bytes: the simple form, or that for few rows; those that do not start on 4: the simple form
    for form in forms.LARGE:
        product("64x64 %s on 4" % form, **dict(forms.SIZES[form], k=1408), scales=4)
    product("thin 4 1 on 4", 60, 1030, 1408, 1, scales=4)
    product("64x64 few on 1", 60, 1030, 2880, 1, scales=1)
    return out


def _main(runtime):
    """In a process of its own, for the real runtime must not be loaded: prints the forms of all calls."""
    lib, out = fake_hip.Lib(runtime), {}
    for key, (name, args) in _calls().items():
        first = lib.fake.fake_notes()
        rc = getattr(lib.lib, name)(*args, 0x1000)
        assert rc == 0 and lib.fake.fake_notes() == first + 1, (key, rc)
        out[key] = _form(lib.fake.fake_name(first).decode())
    print(json.dumps(out))


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    runtime = fake_hip.build(str(tmp_path_factory.mktemp("fake_hip")))
    p = subprocess.run([sys.executable, os.path.abspath(__file__), runtime], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=300)
    assert p.returncode == 0, p.stderr[-2000:]
    return json.loads(p.stdout.splitlines()[-1])


@pytest.mark.parametrize("key", sorted(_calls()))
def test_the_form_that_is_named_runs(launched, key):
    form = launched[key]
    assert key.startswith(form + " "), form


if __name__ == "__main__":
    _main(sys.argv[1])
