"""What the layer norm's and the Muon step's calls launch, without a device: a small library takes the runtime's launches in a
process of its own and writes them down.  Every launch that a valid call leads to is one that the hardware takes, it stays within
the local memory that was asked for, and no launch follows one that was refused."""
import json
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

TAKES = r"""
typedef struct { unsigned x, y, z; } dims;
unsigned long long launches[1024][8];
int launched = 0, fails_at = 0, last = 0, asked = 0, refuses = 0;
static int answer(int e) { if (e) last = e; return e; }
static dims g0, b0;
static unsigned long lds0;
static const void* kernels[4096];
static int most[4096], known = 0;
int __hipPushCallConfiguration(dims grid, dims block, unsigned long lds, void* stream) {
  g0 = grid; b0 = block; lds0 = lds;
  return 0;
}
int __hipPopCallConfiguration(dims* grid, dims* block, unsigned long* lds, void** stream) {
  *grid = g0; *block = b0; *lds = lds0; *stream = 0;
  return 0;
}
int hipFuncSetAttribute(const void* f, int which, int value) {
  asked++;
  if (refuses) return answer(1);
  kernels[known % 4096] = f;
  most[known++ % 4096] = which == 8 ? value : -1;
  return 0;
}
int hipLaunchKernel(const void* f, dims grid, dims block, void** args, unsigned long lds, void* stream) {
  unsigned long long* l = launches[launched++ % 1024];
  l[0] = grid.x; l[1] = grid.y; l[2] = grid.z; l[3] = block.x; l[4] = block.y; l[5] = block.z; l[6] = lds; l[7] = 65536;
  for (int k = 0; k < known && k < 4096; ++k)
    if (kernels[k] == f) l[7] = most[k];
  return answer(launched == fails_at ? 9 : 0);
}
int hipGetLastError(void) { const int e = last; last = 0; return e; }
"""

RUN = r"""
import ctypes, json, sys
takes = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)      # before the library, which binds to it
sys.path.insert(0, sys.argv[2])
from paper_2204_01205_amd import binding as B
lib, p, size = B.lib(), ctypes.c_void_p(1 << 20), ctypes.c_size_t(1 << 62)
seen, names = ((ctypes.c_ulonglong * 8) * 1024).in_dll(takes, "launches"), ("launched", "fails_at", "refuses", "asked")
count, fails, refuses, asked = (ctypes.c_int.in_dll(takes, n) for n in names)

def call(op, kw, fail=0):
    count.value, fails.value, refuses.value, asked.value = 0, max(fail, 0), int(fail < 0), 0
    if op == "muon":
        n = len(kw["tensors"])
        tensors = (B.FnoMuonTensor * max(n, 1))(*[B.FnoMuonTensor(1 << 20, 1 << 20, 1 << 20, b, r, c, k, 1.0, 0.0) for k, b, r, c in kw["tensors"]])
        options = B.FnoMuonOptions(1e-3, 0.9, 1e-7, 3.0, -4.0, 2.0, kw.get("iterations", 5), 1)
        rc = lib.fno_muon_step(n, tensors, ctypes.byref(options), None, 1.0, p, size, None)
    else:
        d = ctypes.byref(B.make_layer_norm_desc(**kw))
        rc = lib.fno_layer_norm_fwd(d, p, p, p, p, None) if op == "fwd" else \
             lib.fno_layer_norm_bwd(d, p, p, p, p, p, p if op == "bwd" else None, p, p, size, None) if op == "no_gx" else \
             lib.fno_layer_norm_bwd(d, p, p, p, p, p, p, p, p, size, None)
    return rc, asked.value, [list(seen[k]) for k in range(min(count.value, 1024))]

out = []
for op, kw, fail in json.loads(sys.stdin.read()):
    out.append(call(op, kw, fail))
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    where = tmp_path_factory.mktemp("launches")
    (where / "takes.c").write_text(TAKES)
    (where / "run.py").write_text(RUN)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(where / "takes.so"), str(where / "takes.c")], check=True)

    def run(calls):
        done = subprocess.run([sys.executable, str(where / "run.py"), str(where / "takes.so"), ROOT], input=json.dumps(calls),
                              capture_output=True, text=True, timeout=300)
        assert done.returncode == 0, done.stderr[-2000:]
        return json.loads(done.stdout.strip().splitlines()[-1])

    return run


def fits(call, made):
    for gx, gy, gz, bx, by, bz, lds, most in made:
        assert 0 < gx * bx < 2 ** 32 and 0 < gy <= 65535 and gz == by == bz == 1 and bx <= 1024 and bx % 64 == 0, (call, made)
        assert lds <= most <= 160 * 1024, (call, made)


def descriptors():
    """Every combination of extremes that the header allows, whatever memory it would take."""
    for layout, widest in ((0, 1024), (1, 16384)):
        for channels in sorted({1, 2, 3, 16, 20, 31, 32, 33, 64, 65, 128, 209, 511, 512, 513, 1024, 2048, 4096, 8191, 16383, 16384}):
            if channels > widest:
                continue
            for batch in (1, 3, 4096, 65535):
                for points in (0, 1, 2, 7, 64, 511, 7200, 70001, 2 ** 21 - 1, 2 ** 31 + 5, 2 ** 40):
                    if batch * channels * points <= 2 ** 44:
                        for dtype in (0, 1):
                            yield dict(batch=batch, channels=channels, npoints=points, layout=layout, dtype=dtype)


def test_every_launch_of_a_norm_is_one_that_the_hardware_takes(launches):
    calls = [(op, kw, 0) for kw in descriptors() for op in ("fwd", "bwd", "no_gx")]
    results = launches(calls)
    assert len(results) == len(calls) > 2000
    for call, (status, _, made) in zip(calls, results):
        empty = call[1]["npoints"] == 0
        assert status == 0 and (bool(made) or empty and call[0] == "fwd"), call
        fits(call, made)


@pytest.mark.parametrize("op", ["fwd", "bwd"])
def test_nothing_is_launched_after_a_launch_of_a_norm_that_failed(launches, op):
    shapes = [dict(batch=b, channels=c, npoints=p, layout=layout) for layout in (0, 1)
              for b, c, p in ((1, 8, 100), (2, 6, 300), (2, 64, 50000), (1, 20, 7000000), (70, 512, 400), (4096, 1024, 2))]
    whole = launches([(op, kw, 0) for kw in shapes])
    calls = [(op, kw, k) for kw, (_, _, made) in zip(shapes, whole) for k in range(1, len(made) + 1)]
    assert len(calls) >= len(shapes)
    for (_, kw, k), (status, _, made) in zip(calls, launches(calls)):
        assert status == -4 and len(made) == k, (kw, k, status, made)


def lists():
    matrices = [(0, b, r, c) for b in (1, 3, 1000) for r in (1, 2, 31, 32, 33, 100, 256) for c in (1, 7, 32, 33, 255, 8192)]
    matrices += [(0, 1, 32768, 32768), (0, 2 ** 31 - 1, 1, 1), (0, 2 ** 31 - 1, 16, 32), (0, 1, 1, 32768), (0, 2 ** 20, 33, 33),
                 (0, 1, 192, 192), (0, 1, 193, 193), (0, 40, 1024, 1024), (0, 1024, 32768, 32)]
    modes = [(1, b, r, c) for b in (1, 17, 7776, 2 ** 31 - 1) for r in (1, 4, 5, 16, 17, 20, 21, 32) for c in (1, 3, 17, 20, 32)
             if b * r * c <= 2 ** 40]
    out = [[m] for m in matrices + modes]
    out += [[], [(0, 0, 5, 5), (1, 3, 0, 4), (0, 2, 3, 0)], [(0, 1, 60, 60)] * 70, [(1, 12, 20, 20)] * 70, [(1, 12, 4, 8)] * 70,
            [(0, 1, 20, 20)] * 70, [(0, 1, 256, 256)] * 33 + [(0, 1, 32, 20)] * 33 + [(1, 64, 20, 20), (1, 64, 30, 20)] * 33]
    return out


@pytest.mark.parametrize("iterations", [0, 1, 5])
def test_every_launch_of_a_step_is_one_that_the_hardware_takes(launches, iterations):
    calls = [("muon", dict(tensors=t, iterations=iterations), 0) for t in lists()]
    for call, (status, _, made) in zip(calls, launches(calls)):
        filled = [t for t in call[1]["tensors"] if min(t[1:]) > 0]
        assert status == 0 and bool(made) == bool(filled), call
        fits(call, made)


def test_nothing_is_launched_after_a_launch_of_a_step_that_failed(launches):
    mixed = [[(0, 1, 60, 60)], [(0, 3, 20, 20)], [(1, 9, 20, 20)], [(1, 9, 4, 5)],
             [(0, 1, 60, 60), (1, 9, 20, 20), (0, 1, 20, 20), (1, 9, 32, 32), (0, 2, 300, 1000)]]
    whole = launches([("muon", dict(tensors=t), 0) for t in mixed])
    calls = [("muon", dict(tensors=t), k) for t, (_, _, made) in zip(mixed, whole) for k in range(1, len(made) + 1)]
    assert len(calls) > 30
    for (_, kw, k), (status, _, made) in zip(calls, launches(calls)):
        assert status == -4 and len(made) == k, (kw, k, status, len(made))


def test_a_refused_size_of_local_memory_is_an_error(launches):
    """Kernels that need more than 64 KB ask the runtime first: where it refuses, the call fails and that kernel is not launched."""
    calls = [("muon", dict(tensors=[t]), -1) for t in ((1, 9, 20, 20), (1, 9, 32, 32), (0, 1, 32, 256), (0, 1, 8, 8))]
    calls += [("bwd", dict(batch=1, channels=c, npoints=5000, layout=1), -1) for c in (16, 512)]
    for call, (status, asked, made) in zip(calls, launches(calls)):
        assert (status == -4 and not made) if asked else (status == 0 and made), call
        assert all(l[6] <= 65536 for l in made), call
