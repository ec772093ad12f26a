"""What the 4-bit operators and the balance loss do at the ends of the sizes they take, and when a launch is refused, on a runtime that runs nothing
(fake_hip_limits.cpp)."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
A = 0x7000000000                                                 # an address that is never used

QUANTISE = dict(x=A, type=1, ldx=1, rows=4, cols=1, act=0, slots=None, copies=1, out=4, q=A, ldq=1, s=A, lds=1)
COLUMNS = dict(x=A, type=1, ldx=1, rows=4, cols=1, g=None, groups=1, q=A, ldq=1 << 31, s=A, lds=1 << 27)
READ = dict(q=A, ldq=1, s=A, lds=1, rows=4, cols=1, x=A, type=1, ldx=1)
MATMUL = dict(x=A, ldx=1, xs=A, lxs=1, w=A, ldw=1, wg=0, ws=A, lws=1, wsg=0, g=None, groups=1, y=A, yt=1, ldy=1, m=4, n=1, k=1)
GRAD_W = dict(a=A, la=64, sa=A, lsa=4, b=A, lb=64, sb=A, lsb=4, g=None, groups=1, dw=A, dt=1, ld=1, dg=0, m=4, n=1, k=1)
BALANCE = dict(l=A, type=1, ld=2, n=4, e=2, ex=A, k=1, g=None, groups=1, c=A, t=A, s=A, loss=A, ws=A, size=1 << 40)
BALANCE_GRAD = dict(l=A, type=1, ld=2, n=4, e=2, g=None, groups=1, c=A, t=A, dl=A, flags=0, out=A, ldo=2)
FEW = dict(x=A, ldx=64, n=4, h=64, l=A, lt=0, ldl=8, e=8, k=2, flags=1, w1=A, s1=A, w2=A, s2=A, f=48, wt=4, kind=1, out=A, ot=1, ldo=64, ws=A, size=1 << 40)

# (name, arguments, the size that grows, the largest that is taken)
GROWING = [("tuna_fp4_quantize", QUANTISE, "rows", (1 << 31) - 1),
           ("tuna_fp4_dequantize", READ, "rows", (1 << 31) - 1),
           ("tuna_fp4_quantize_columns", COLUMNS, "rows", 128 * ((1 << 24) - 1)),
           ("tuna_fp4_matmul", MATMUL, "m", 64 * ((1 << 24) - 1)),
           ("tuna_fp4_matmul_grad_w", GRAD_W, "n", 64 * ((1 << 24) - 1)),
           ("tuna_moe_balance", BALANCE, "n", 1 << 28),
           ("tuna_moe_balance_grad", BALANCE_GRAD, "n", 1 << 28)]


def _main(runtime):
    """In a process of its own, for the real runtime must not be loaded: prints the results of all calls."""
    fake = ctypes.CDLL(runtime, mode=ctypes.RTLD_GLOBAL)
    sys.path.insert(0, os.path.dirname(HERE))
    import paper_2411_02581_amd.binding as b
    lib, out = b.load(), {}

    def do(key, name, args, refuse=-1):
        fake.fake_refuse(refuse)
        rc = getattr(lib, name)(*args.values(), 0x1000)
        out[key] = [{b.TUNA_OK: "ok", b.TUNA_ERR_TOO_LARGE: "large", b.TUNA_ERR_HIP: "hip"}.get(rc, rc), fake.fake_asked(), fake.fake_taken()]

    for name, args, what, most in GROWING:
        size = {what: most}
        if name == "tuna_fp4_quantize":
            size["out"] = most
        do(name + " most", name, dict(args, **size))
        do(name + " more", name, dict(args, **{k: v + 1 for k, v in size.items()}))
        do(name + " end", name, dict(args, **{k: 1 << 31 for k in size}))
    # wide rows on the way to the limit of a grid of tiles, and behind it
    for m in (1 << 20, (1 << 30) - 64):
        do("tiles %d" % m, "tuna_fp4_matmul", dict(MATMUL, ldx=16, lxs=4, ldw=16, lws=4, m=m, n=80, ldy=80, k=32))
    for refuse in range(-1, 4):
        do("balance %d" % refuse, "tuna_moe_balance", dict(BALANCE, n=1000), refuse)
        do("few %d" % refuse, "tuna_moe_few", FEW, refuse)
    print(json.dumps(out))


@pytest.fixture(scope="module")
def results(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("fake_hip_fp4") / "libamdhip64.so.7")
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
    for m in (1 << 20, (1 << 30) - 64):
        assert results["tiles %d" % m] == ["ok", 1, 1]


def test_nothing_follows_a_refused_launch(results):
    """The kernels behind one that was refused would read what it did not write."""
    launches = results["balance -1"][1]
    assert results["balance -1"] == ["ok", launches, launches] and results["few -1"] == ["ok", 2, 2]
    for n in range(4):
        assert results["balance %d" % n] == (["hip", n + 1, n] if n < launches else ["ok", launches, launches]), n
        assert results["few %d" % n] == (["hip", n + 1, n] if n < 2 else ["ok", 2, 2]), n


if __name__ == "__main__":
    _main(sys.argv[1])
