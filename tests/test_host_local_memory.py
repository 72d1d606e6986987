"""What kernels of the Muon step ask of the runtime before they take more than 64 KB of local memory a block, without a device.  The
request holds for the whole process: one that depended on the call's sizes could be lowered by another thread between a call's request and its
launch.  So a kernel asks for the same whatever it is launched with, and never for less than that."""
import json
import shutil
import subprocess
import sys

import pytest

from test_host_layer_norm_muon_launches import ROOT, TAKES

RUN = r"""
import ctypes, json, sys
takes = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)      # before the library, which binds to it
sys.path.insert(0, sys.argv[2])
from paper_2204_01205_amd import binding as B
lib, p, size = B.lib(), ctypes.c_void_p(1 << 20), ctypes.c_size_t(1 << 62)
launched, known = (ctypes.c_int.in_dll(takes, n) for n in ("launched", "known"))
functions, launches = (ctypes.c_void_p * 1024).in_dll(takes, "functions"), ((ctypes.c_ulonglong * 8) * 1024).in_dll(takes, "launches")
asking, asked = (ctypes.c_void_p * 4096).in_dll(takes, "kernels"), (ctypes.c_int * 4096).in_dll(takes, "most")
out = []
for kind, batch, rows, cols in json.loads(sys.stdin.read()):
    launched.value = known.value = 0
    options = B.FnoMuonOptions(1e-3, 0.9, 1e-7, 3.0, -4.0, 2.0, 5, 1)
    tensor = B.FnoMuonTensor(1 << 20, 1 << 20, 1 << 20, batch, rows, cols, kind, 1.0, 0.0)
    assert lib.fno_muon_step(1, ctypes.byref(tensor), ctypes.byref(options), None, 1.0, p, size, None) == 0
    out.append(([(asking[k], asked[k]) for k in range(known.value)], [(functions[k], launches[k][6]) for k in range(launched.value)]))
print(json.dumps(out))
"""


def test_a_kernel_asks_for_the_same_whatever_it_is_launched_with(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    taken = TAKES.replace("int launched = 0,", "const void* functions[1024];\nint launched = 0,")
    taken = taken.replace("unsigned long long* l = launches", "functions[launched % 1024] = f;\n  unsigned long long* l = launches")
    taken = taken.replace("static const void* kernels", "const void* kernels").replace("static int most[4096], known", "int most[4096], known")
    (tmp_path / "takes.c").write_text(taken)
    (tmp_path / "run.py").write_text(RUN)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(tmp_path / "takes.so"), str(tmp_path / "takes.c")], check=True)
    calls = [(1, 40, rows, cols) for rows in range(1, 33) for cols in range(rows, 33)]
    calls += [(0, 1, m, n) for m in range(1, 33) for n in sorted({m, 100, 200, 256, 400, 500, 512, 546, 700, 2000, 16384 // m}) if m * n <= 16384]
    done = subprocess.run([sys.executable, str(tmp_path / "run.py"), str(tmp_path / "takes.so"), ROOT], input=json.dumps(calls),
                          capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    requests, most, large = {}, {}, 0
    for call, (asked, launched) in zip(calls, json.loads(done.stdout.strip().splitlines()[-1])):
        for kernel, size in asked:
            requests.setdefault(kernel, set()).add(size)
        for kernel, size in launched:
            most[kernel] = max(size, most.get(kernel, 0))
            if size > 65536:
                large += 1
                assert kernel in dict(asked), call
    assert large > 100 and len(requests) >= 6                # 4 to 8 tiles of spectral weights, and the small matrices
    for kernel, sizes in requests.items():
        assert len(sizes) == 1 and most[kernel] <= min(sizes) <= 160 * 1024, (sizes, most[kernel])
