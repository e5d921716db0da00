"""The host arithmetic of the losses and gradient lists (space_train_plan.h) on the CPU, and what the binding refuses before it calls."""
import ctypes
import os
import random
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2402_11809_amd", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src = d / "plan.cpp"
    src.write_text('''#include "space_train_plan.h"
using namespace space;
extern "C" int apart(uint64_t x, int64_t xs, uint64_t d, int64_t ds, int64_t rows, int64_t cols, int64_t bytes) {
    return rows_apart(x, xs, d, ds, rows, cols, bytes);
}
extern "C" int written(uint64_t* v, int n) {  // (lo, hi, written) each
    ByteRange r[64];
    for (int i = 0; i < n; ++i) r[i] = ByteRange{(uintptr_t)v[3 * i], (uintptr_t)v[3 * i + 1], v[3 * i + 2] != 0};
    return written_apart(r, n);
}
''')
    so = d / "plan.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.apart.argtypes = [ctypes.c_uint64, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64]
    lib.written.argtypes = [ctypes.POINTER(ctypes.c_uint64), ctypes.c_int]
    return lib


def test_rows_apart_never_calls_meeting_rows_apart(lib):
    rng = random.Random(0)
    yes = 0
    for _ in range(3000):
        rows, cols, b = rng.randint(1, 5), rng.randint(1, 9), rng.choice([2, 4])
        xs, ds = cols + rng.randint(0, 12), cols + rng.randint(0, 12)
        if rng.random() < 0.6:
            ds = xs
        x, d = 1000 * b, (1000 + rng.randint(-60, 60)) * b
        bytes_of = lambda p, s: {p + (r * s + c) * b + i for r in range(rows) for c in range(cols) for i in range(b)}
        meet = bool(bytes_of(x, xs) & bytes_of(d, ds))
        got = lib.apart(x, xs, d, ds, rows, cols, b)
        assert not (got and meet), (x, xs, d, ds, rows, cols, b)
        if xs == ds and rows > 1 and not meet and abs(x - d) // b < xs:
            assert got  # side by side
        yes += got
    assert yes > 500


def test_written_ranges_against_a_count_of_bytes(lib):
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(5000):
        n = rng.randint(0, 5)
        rs = [(lo, lo + rng.randint(1, 12), rng.randint(0, 1)) for lo in (rng.randint(1, 60) for _ in range(n))]
        meet = any((a[2] or b[2]) and a[0] < b[1] and b[0] < a[1] for i, a in enumerate(rs) for b in rs[:i])
        v = (ctypes.c_uint64 * (3 * n + 1))(*[w for r in rs for w in r])
        assert lib.written(v, n) == (not meet), rs
        seen[meet] += 1
    assert min(seen) > 500


def test_structs_match_the_header(tmp_path):
    from paper_2402_11809_amd import binding
    text = open(os.path.join(ROOT, "include", "space.h")).read()
    structs = {"space_loss_io": binding.SpaceLossIO, "space_policy_params": binding.SpacePolicyParams,
               "space_preference_params": binding.SpacePreferenceParams, "space_grad_tensor": binding.SpaceGradTensor}
    for name, cls in structs.items():
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        assert [re.findall(r"(\w+)\s*$", d.strip())[0] for d in body.split(";") if d.strip()] == [f[0] for f in cls._fields_], name
    src = tmp_path / "sizes.c"
    src.write_text('#include "space.h"\n#include <stdio.h>\nint main(void) {\n' + "".join(f'    printf("%zu\\n", sizeof({n}));\n' for n in structs) +
                   '    printf("%d %d\\n", SPACE_LOSS_WORK, SPACE_GRAD_WORK);\n    return 0;\n}\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(c) for c in structs.values()] + [binding.SPACE_LOSS_WORK, binding.SPACE_GRAD_WORK]


def test_calls_without_a_context_are_refused_and_do_not_crash():
    from paper_2402_11809_amd import binding
    lib = binding.load_library()
    io, pol, pref = binding.SpaceLossIO(), binding.SpacePolicyParams(), binding.SpacePreferenceParams()
    E = binding.SPACE_EINVAL
    assert lib.space_sar_loss_grad(None, ctypes.byref(io), None) == E
    assert lib.space_policy_loss(None, ctypes.byref(io), ctypes.byref(pol), None) == E
    assert lib.space_preference_loss(None, ctypes.byref(io), ctypes.byref(pref), None) == E
    assert lib.space_grad_norm(None, None, 0, None, None, None) == E
    assert lib.space_grad_clip(None, None, 0, None, 1.0, None) == E


def test_dense_tensors_are_told_from_others():
    torch = pytest.importorskip("torch")
    from paper_2402_11809_amd import binding
    t = torch.zeros(4, 6)
    for good in (t, t.t(), t.view(4, 1, 6), t[:1], t[:, :0], torch.zeros(()), torch.zeros(2, 3, 5).permute(1, 2, 0), t.expand(1, 4, 6)):
        assert binding._dense(good), good.shape
    for bad in (t[:, :3], t[::2], t[:1].expand(4, 6), t[:, 1:2]):
        assert not binding._dense(bad), bad.shape
    assert binding._same_order(t, torch.ones(4, 6)) and not binding._same_order(t, torch.ones(6, 4).t())
    assert binding._row_stride(t[:, :3]) == 6 and binding._row_stride(t[:1, :3]) >= 3 and binding._row_stride(None) == 0


def test_rows_that_meet_a_range_against_a_count_of_bytes(tmp_path):
    src = tmp_path / "meet.cpp"
    src.write_text('''#include "space_train_plan.h"
extern "C" int meet(uint64_t x, int64_t xs, int64_t rows, int64_t cols, int64_t bytes, uint64_t lo, uint64_t hi) {
    return space::rows_meet(x, xs, rows, cols, bytes, lo, hi);
}
''')
    so = tmp_path / "meet.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.meet.argtypes = [ctypes.c_uint64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_uint64, ctypes.c_uint64]
    rng = random.Random(2)
    seen = [0, 0]
    for _ in range(5000):
        rows, cols, b = rng.randint(1, 5), rng.randint(1, 9), rng.choice([2, 4])
        xs = cols + rng.choice([0, rng.randint(0, 12)])
        x, lo = 500, 500 + rng.randint(-40, rows * xs * b + 20)
        hi = lo + rng.randint(1, 24)
        held = {x + (r * xs + c) * b + i for r in range(rows) for c in range(cols) for i in range(b)}
        want = not held.isdisjoint(range(lo, hi))
        assert lib.meet(x, xs, rows, cols, b, lo, hi) == want, (xs, rows, cols, b, lo, hi)
        seen[want] += 1
    assert min(seen) > 500
    # the last row of a large buffer, and the gap in front of it
    x, xs, rows, cols = 1 << 44, (1 << 26) + 3, 4000000, 1001
    last = x + (rows - 1) * xs * 2
    assert lib.meet(x, xs, rows, cols, 2, last + 2 * cols - 1, last + 2 * cols + 9) and not lib.meet(x, xs, rows, cols, 2, last + 2 * cols, last + 2 * cols + 9)
    assert lib.meet(x, xs, rows, cols, 2, last - 1, last + 1) and not lib.meet(x, xs, rows, cols, 2, last - 9, last)


def test_ranges_that_meet_against_a_count_of_bytes(tmp_path):
    src = tmp_path / "pair.cpp"
    src.write_text('''#include "space_train_plan.h"
extern "C" int meet(uint64_t a, uint64_t an, uint64_t b, uint64_t bn) { return space::ranges_meet(a, an, b, bn); }
''')
    so = tmp_path / "pair.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.meet.argtypes = [ctypes.c_uint64] * 4
    for a in range(6):
        for an in range(5):
            for b in range(6):
                for bn in range(5):
                    assert lib.meet(a, an, b, bn) == (not set(range(a, a + an)).isdisjoint(range(b, b + bn))), (a, an, b, bn)
