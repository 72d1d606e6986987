"""What the group norm's and the optimizer's calls launch, without a device: a small library takes the runtime's launches in a
process of its own and writes them down.  Every launch that a valid descriptor leads to is one that the hardware takes, and no launch
follows one that was refused."""
import json
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

TAKES = r"""
typedef struct { unsigned x, y, z; } dims;
unsigned long long launches[256][7];
int launched = 0, fails_at = 0, last = 0;
static int answer(int e) { if (e) last = e; return e; }
static dims g0, b0;
static unsigned long lds0;
int __hipPushCallConfiguration(dims grid, dims block, unsigned long lds, void* stream) {
  g0 = grid; b0 = block; lds0 = lds;
  return 0;
}
int __hipPopCallConfiguration(dims* grid, dims* block, unsigned long* lds, void** stream) {
  *grid = g0; *block = b0; *lds = lds0; *stream = 0;
  return 0;
}
int hipLaunchKernel(const void* f, dims grid, dims block, void** args, unsigned long lds, void* stream) {
  unsigned long long* l = launches[launched++ % 256];
  l[0] = grid.x; l[1] = grid.y; l[2] = grid.z; l[3] = block.x; l[4] = block.y; l[5] = block.z; l[6] = lds;
  return answer(launched == fails_at ? 9 : 0);
}
int hipGetLastError(void) { const int e = last; last = 0; return e; }
"""

RUN = r"""
import ctypes, json, sys
takes = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)      # before the library, which binds to it
sys.path.insert(0, sys.argv[2])
from paper_2204_01205_amd import binding as B
lib, p, size = B.lib(), ctypes.c_void_p(1 << 20), ctypes.c_size_t(1 << 60)
seen, count, fails = (((ctypes.c_ulonglong * 7) * 256).in_dll(takes, "launches"), ctypes.c_int.in_dll(takes, "launched"),
                      ctypes.c_int.in_dll(takes, "fails_at"))

def call(op, kw, fail=0):
    count.value, fails.value = 0, fail
    if "sizes" in kw:
        n, bits = len(kw["sizes"]), kw["bits"]
        tensors = (B.FnoAdamwTensor * max(n, 1))(*[B.FnoAdamwTensor(1 << 20, 1 << 20, 1 << 20, 1 << 20, 1 << 20, s, 0.0) for s in kw["sizes"]])
        outs = (ctypes.c_void_p * max(n, 1))(*[1 << 20] * n)
        rc = lib.fno_adamw_step(n, tensors, bits, 1e-3, 0.9, 0.999, 1e-8, 1, None, 1.0, 0, None) if op == "step" else \
             lib.fno_grad_norm(n, tensors, p, p, size, None) if op == "norm" else \
             lib.fno_adamw_state_read(n, tensors, outs, outs, None)
        return rc, [list(seen[k]) for k in range(min(count.value, 256))]
    d = ctypes.byref(B.make_norm_desc(**kw))
    rc = lib.fno_group_norm_fwd(d, p, p, p, p, p, p, p, size, None) if op == "fwd" else \
         lib.fno_group_norm_bwd(d, p, p, p, p, p, p, p, p, p, p, size, None)
    return rc, [list(seen[k]) for k in range(count.value)]

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


def descriptors():
    """Every combination of extremes that the header allows, whatever memory it would take."""
    for batch, channels in ((1, 1), (1, 1024), (3, 20), (4096, 1024), (8192, 1024), (65535, 128), (65535, 1), (40000, 209)):
        for groups in sorted({1, channels} | {g for g in (2, 11, 64, 512) if channels % g == 0}):
            for points in (0, 1, 2, 7, 100, 511, 512, 7200, 8192, 16384, 70001, 2 ** 21 - 1, 2 ** 31 + 5, 2 ** 40):
                if batch * channels * points > 2 ** 44:
                    continue
                for layout in (0, 1):
                    for dtype in (0, 1):
                        yield dict(batch=batch, channels=channels, groups=groups, npoints=points, layout=layout, dtype=dtype)


def test_every_launch_is_one_that_the_hardware_takes(launches):
    calls = [(op, kw, 0) for kw in descriptors() for op in ("fwd", "bwd")]
    results = launches(calls)
    assert len(results) == len(calls) > 1000
    for call, (status, made) in zip(calls, results):
        assert status == 0 and made, call
        for gx, gy, gz, bx, by, bz, lds in made:
            assert 0 < gx * bx < 2 ** 32 and 0 < gy <= 65535 and gz == by == bz == 1 and bx <= 1024 and bx % 64 == 0, (call, made)
            assert lds <= 150 * 1024, (call, made)       # 160 KB with the kernels' own arrays


@pytest.mark.parametrize("op", ["fwd", "bwd"])
def test_nothing_is_launched_after_a_launch_that_failed(launches, op):
    shapes = [dict(batch=b, channels=c, groups=g, npoints=p, layout=layout) for layout in (0, 1)
              for b, c, g, p in ((1, 8, 2, 100), (2, 6, 3, 300), (2, 8, 2, 50000), (1, 20, 4, 7000000), (70, 64, 1, 400), (4096, 1024, 1024, 2))]
    whole = launches([(op, kw, 0) for kw in shapes])
    calls = [(op, kw, k) for kw, (_, made) in zip(shapes, whole) for k in range(1, len(made) + 1)]
    assert max(k for _, _, k in calls) >= 3
    for (_, kw, k), (status, made) in zip(calls, launches(calls)):
        assert status == -4 and len(made) == k, (kw, k, status, made)


LISTS = [[1], [0, 5, 0], [4096, 4097, 1], [7] * 200, [0] * 70 + [3], [2 ** 22] * 65, [2 ** 32 + 777, 12], [2 ** 40, 2 ** 40, 1, 2 ** 39], [2 ** 34] * 130]


@pytest.mark.parametrize("op,bits", [("step", 32), ("step", 8), ("norm", 32), ("read", 8)])
def test_lists_of_tensors(launches, op, bits):
    whole = launches([(op, dict(sizes=s, bits=bits), 0) for s in LISTS])
    calls = []
    for sizes, (status, made) in zip(LISTS, whole):
        assert status == 0 and made, sizes
        for gx, gy, gz, bx, by, bz, lds in made:
            assert 0 < gx * bx < 2 ** 32 and gy == gz == by == bz == 1 and bx <= 1024 and lds == 0, (sizes, made)
        # up to 64 tensors a launch
        assert len(made) <= -(-len(sizes) // 64) + (op == "norm") + sum(n > 2 ** 32 for n in sizes)
        calls += [(op, dict(sizes=sizes, bits=bits), k) for k in range(1, len(made) + 1)]
    for (_, kw, k), (status, made) in zip(calls, launches(calls)):
        assert status == -4 and len(made) == k, (kw["sizes"][:5], k)
