"""Which kernels the Muon step and the layer norm launch, by their names, without a device: a small library takes the runtime's
registrations and launches in a process of its own.  The lists that stand for tiles of 128 take them, and those on the other side of each
limit do not; every kernel that is built is one that a call can reach."""
import json
import shutil
import subprocess
import sys

import pytest

from test_gpu_muon_dense import AT_LEAST, BELOW, IN_128, IN_64
from test_host_layer_norm_muon_launches import ROOT, TAKES

NAMES = r"""
const char* names[8192];
const void* owners[8192];
int registered = 0;
void __hipRegisterFunction(void** modules, const void* f, char* symbol, const char* name, unsigned limit, void* tid, void* bid, void* block,
                           void* grid, int* wave) {
  owners[registered % 8192] = f;
  names[registered++ % 8192] = name;
}
"""

RUN = r"""
import ctypes, json, sys
takes = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)      # before the library, which binds to it
sys.path.insert(0, sys.argv[2])
from paper_2204_01205_amd import binding as B
registered = ctypes.c_int.in_dll(takes, "registered")
registered.value = 0                                          # torch's own kernels
lib = B.lib()
count = ctypes.c_int.in_dll(takes, "launched")
functions = (ctypes.c_void_p * 1024).in_dll(takes, "functions")
names = dict(zip((ctypes.c_void_p * 8192).in_dll(takes, "owners"), (ctypes.c_char_p * 8192).in_dll(takes, "names")))
assert 0 < registered.value < 8192
p, out = ctypes.c_void_p(1 << 20), []
for call in json.loads(sys.stdin.read()):
    count.value, size = 0, ctypes.c_size_t(1 << 62)
    if isinstance(call, dict):
        desc = ctypes.byref(B.make_layer_norm_desc(**call))
        status = lib.fno_layer_norm_fwd(desc, p, p, p, p, None) or lib.fno_layer_norm_bwd(desc, p, p, p, p, p, p, p, p, size, None)
    else:
        array = (B.FnoMuonTensor * len(call))(*[B.FnoMuonTensor(1 << 20, 1 << 20, 1 << 20, b, r, c, k, 1.0, 0.0) for k, b, r, c in call])
        options = B.FnoMuonOptions(1e-3, 0.9, 1e-7, 3.0, -4.0, 2.0, 5, 1)
        status = lib.fno_muon_step(len(call), array, ctypes.byref(options), None, 1.0, p, size, None)
    assert status == 0 and count.value <= 1024
    out.append([names[functions[k]].decode() for k in range(count.value)])
out.append([n.decode() for n in names.values() if n])
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    where = tmp_path_factory.mktemp("kernels")
    taken = TAKES.replace("int launched = 0,", "const void* functions[1024];\nint launched = 0,")
    taken = taken.replace("unsigned long long* l = launches", "functions[launched % 1024] = f;\n  unsigned long long* l = launches")
    (where / "takes.c").write_text(taken + NAMES)
    (where / "run.py").write_text(RUN)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(where / "takes.so"), str(where / "takes.c")], check=True)

    def run(calls, built=False):
        """Names of the launched kernels: of a Muon step of a list of (kind, batch, rows, cols), or a layer norm's two passes with a
        dictionary's descriptor.  built: of all kernels of the library behind them."""
        done = subprocess.run([sys.executable, str(where / "run.py"), str(where / "takes.so"), ROOT], input=json.dumps(calls),
                              capture_output=True, text=True, timeout=300)
        assert done.returncode == 0, done.stderr[-2000:]
        names = json.loads(done.stdout.strip().splitlines()[-1])
        return names if built else names[:-1]

    return run


def tensors(shapes):
    """(kind, batch, rows, cols) of a list of (shape, is_complex)."""
    out = []
    for shape, is_complex in shapes:
        rows, cols = shape[:2] if is_complex else shape[-2:]
        batch = 1
        for n in shape[2:] if is_complex else shape[:-2]:
            batch *= n
        out.append((int(is_complex), batch, rows, cols))
    return out


def tile_sizes(names):
    return {t for n in names for t in (64, 128) if f"dense_product_kernelILi{t}E" in n}


def summed(names, tile):
    return any(f"dense_sum_kernelILi{tile}E" in n for n in names)


def test_lists_on_either_side_of_the_tiles_of_128(kernels):
    which = sorted(IN_128)
    got = dict(zip(which, kernels([tensors(IN_128[k]) for k in which])))
    for k in which:
        assert tile_sizes(got[k]) == ({64, 128} if k == "mixed" else {128}), k
        assert all(any(f"dense_product_kernelILi128ELi{phase}E" in n for n in got[k]) for phase in range(3)), k
    # with sums that are split and sums that are not
    assert summed(got["wide"], 128) and summed(got["mixed"], 128) and summed(got["mixed"], 64) and not summed(got["stack"], 128)
    assert all(any(f"dense_sum_kernelILi128ELi{phase}E" in n for n in got["one"]) for phase in range(3))
    below, at_least = kernels([tensors(BELOW), tensors(AT_LEAST)])
    assert tile_sizes(below) == {64} and tile_sizes(at_least) == {128}
    for names in kernels([tensors([(shape, False)]) for shape in IN_64]):
        assert tile_sizes(names) == {64}


def test_a_short_side_of_192_stays_with_tiles_of_64(kernels):
    inside, beyond, thin = kernels([[(0, 1000, 192, 192)], [(0, 1000, 193, 193)], [(0, 100, 20, 40), (0, 1, 20, 20)]])
    assert tile_sizes(inside) == {64} and tile_sizes(beyond) == {128} and tile_sizes(thin) == set()


KERNELS = ("first_fwd_kernel", "first_bwd_kernel", "shared_fwd_kernel", "shared_bwd_kernel", "tile_fwd_kernel", "tile_bwd_kernel",
           "wide_fwd_kernel", "wide_bwd_kernel", "layer_sum_kernel", "muon_modes_kernel", "muon_modes2_kernel", "muon_modes5_kernel",
           "muon_small_kernel", "dense_momentum_kernel", "dense_parts_kernel", "dense_product_kernel", "dense_sum_kernel")
kind_of = lambda name: next((k for k in KERNELS if f"{len(k)}{k}" in name), None)


def test_every_kernel_that_is_built_can_be_reached(kernels):
    calls = [dict(batch=1, channels=c, npoints=points, layout=layout, dtype=dtype, activation=act)
             for layout, widths in ((0, [1, 8, 9, 12, 13, 16, 17, 20, 21, 24, 25, 32, 128, 129, 256, 257, 512, 513, 1024]),
                                    (1, list(range(1, 65)) + [128, 256, 480, 511, 512, 513, 1000, 1024, 1500, 2048, 3000, 4096, 5000, 8192, 9000, 16384]))
             for c in widths for points in (10, 2 ** 18, 2 ** 29 // c) for dtype in (0, 1) for act in (0, 1, 2)]
    calls += [tensors(shapes) for shapes in IN_128.values()] + [tensors([(shape, False)]) for shape in IN_64]
    calls += [[(1, 100, rows, cols)] for rows in range(1, 33) for cols in (rows, 32)] + [[(1, 100000, 8, 8)]]
    *launched, built = kernels(calls, built=True)
    reached, built = {n for names in launched for n in names}, {n for n in built if kind_of(n)}
    assert {kind_of(n) for n in built} == set(KERNELS) and len(built) > 200
    assert not built - reached, sorted(built - reached)
