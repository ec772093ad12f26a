"""What include/tuna_moe.h does at the ends of the sizes it takes, and when a launch is refused, on a runtime that runs nothing (fake_hip_limits.cpp)."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
A = 0x7000000000                                                 # an address that is never used

ROUTE = dict(logits=A, type=1, ld=2, n=4, e=2, k=1, flags=0, experts=A, weights=A, slots=A, rows=A, row_bytes=1, sc=None, sd=None, rc=None, rd=None, ws=A,
             size=1 << 40)
ROUTE_GRAD = dict(logits=A, type=1, ld=2, n=4, e=2, k=1, flags=0, experts=A, weights=A, dw=A, dl=A, ldd=2)
QUANTISE = dict(x=A, type=1, ldx=1, rows=4, cols=1, act=0, slots=None, copies=1, out=4, q=A, ldq=1, s=A, lds=1, kind=1)
COLUMNS = dict(x=A, type=1, ldx=1, rows=4, cols=1, g=None, groups=1, q=A, ldq=1 << 31, s=A, lds=1 << 24, kind=1)
MATMUL = dict(x=A, ldx=1, xs=A, lxs=1, w=A, ldw=1, wg=0, ws=A, lws=1, wsg=0, kind=1, g=None, groups=1, y=A, yt=1, ldy=1, m=4, n=1, k=1)
GRAD_W = dict(a=A, la=128, sa=A, lsa=1, b=A, lb=128, sb=A, lsb=1, kind=1, g=None, groups=1, dw=A, dt=1, ld=1, dg=0, m=4, n=1, k=1)
COMBINE = dict(y=A, yt=1, ldy=1, rows=8, slots=A, w=A, n=4, k=1, cols=1, out=A, ot=1, ldo=1)
COMBINE_GRAD = dict(d=A, ot=1, ldd=1, y=A, yt=1, ldy=1, rows=8, slots=A, w=A, n=4, k=1, cols=1, dy=A, lddy=1, dw=A)
FEW = dict(x=A, ldx=64, n=4, h=64, l=A, lt=0, ldl=8, e=8, k=2, flags=1, w1=A, s1=A, w2=A, s2=A, f=48, wt=2, kind=0, out=A, ot=1, ldo=64, ws=A, size=1 << 40)

# (name, arguments, the size that grows, the largest that is taken): as many blocks of threads as fit 2^32 - 1 threads
GROWING = [("tuna_moe_route", ROUTE, "n", 4 * ((1 << 24) - 1)),
           ("tuna_moe_route_grad", ROUTE_GRAD, "n", 4 * ((1 << 24) - 1)),
           ("tuna_fp8_quantize", QUANTISE, "rows", 32 * ((1 << 24) - 1)),
           ("tuna_fp8_quantize_columns", COLUMNS, "rows", 128 * ((1 << 24) - 1)),
           ("tuna_fp8_matmul", MATMUL, "m", 64 * ((1 << 24) - 1)),
           ("tuna_fp8_matmul_grad_w", GRAD_W, "n", 64 * ((1 << 24) - 1)),
           ("tuna_moe_combine_grad", COMBINE_GRAD, "n", (1 << 24) - 1)]


def _call(lib, name, args):
    return getattr(lib, name)(*args.values(), 0x1000)


def _main(runtime):
    """In a process of its own, for the real runtime must not be loaded: prints the results of all calls."""
    fake = ctypes.CDLL(runtime, mode=ctypes.RTLD_GLOBAL)
    sys.path.insert(0, os.path.dirname(HERE))
    import paper_2411_02581_amd.binding as b
    lib, out = b.load(), {}

    def do(key, name, args, refuse=-1):
        fake.fake_refuse(refuse)
        rc = _call(lib, name, args)
        out[key] = [{b.TUNA_OK: "ok", b.TUNA_ERR_TOO_LARGE: "large", b.TUNA_ERR_HIP: "hip"}.get(rc, rc), fake.fake_asked(), fake.fake_taken()]

    for name, args, what, most in GROWING:
        size = {what: most}
        if name == "tuna_fp8_quantize":
            size["out"] = most
        do(name + " most", name, dict(args, **size))
        more = {k: v + 1 for k, v in size.items()}
        do(name + " more", name, dict(args, **more))
        do(name + " end", name, dict(args, **{k: (1 << 31) - 1 for k in size}))
    do("combine", "tuna_moe_combine", dict(COMBINE, n=32768 * 65535))
    # tiles of 128 x 128 on the way to the limit of their grid, and behind it: the simple form
    for m in (1 << 20, (1 << 30) - 1):
        do("tiles %d" % m, "tuna_fp8_matmul", dict(MATMUL, ldx=16, ldw=16, m=m, n=80, ldy=80, k=16))
    for refuse in range(-1, 5):
        do("route %d" % refuse, "tuna_moe_route", dict(ROUTE, n=100), refuse)
        do("few %d" % refuse, "tuna_moe_few", FEW, refuse)
    print(json.dumps(out))


@pytest.fixture(scope="module")
def results(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("fake_hip_limits") / "libamdhip64.so.7")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + HERE, "-Wl,-soname,libamdhip64.so.7",
                    "-o", lib, os.path.join(HERE, "fake_hip_limits.cpp")], check=True)
    p = subprocess.run([sys.executable, os.path.abspath(__file__), lib], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=300)
    assert p.returncode == 0, p.stderr[-2000:]
    return json.loads(p.stdout.splitlines()[-1])


@pytest.mark.parametrize("name", [g[0] for g in GROWING])
def test_sizes_beyond_a_grid_are_refused_before_anything_is_enqueued(results, name):
    rc, asked, taken = results[name + " most"]
    assert rc == "ok" and asked == taken >= 1
    assert results[name + " more"] == ["large", 0, 0]
    assert results[name + " end"] == ["large", 0, 0]


def test_large_sizes_that_fit_are_taken(results):
    assert results["combine"] == ["ok", 1, 1]
    assert results["tiles %d" % (1 << 20)] == ["ok", 1, 1]
    assert results["tiles %d" % ((1 << 30) - 1)] == ["ok", 1, 1]


def test_nothing_follows_a_refused_launch(results):
    """The kernels behind one that was refused would read what it did not write."""
    assert results["route -1"] == ["ok", 4, 4] and results["few -1"] == ["ok", 2, 2]
    for n in range(5):
        assert results["route %d" % n] == (["hip", n + 1, n] if n < 4 else ["ok", 4, 4]), n
        assert results["few %d" % n] == (["hip", n + 1, n] if n < 2 else ["ok", 2, 2]), n


if __name__ == "__main__":
    _main(sys.argv[1])
