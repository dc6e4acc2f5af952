"""Which kernels the loss over a vocabulary takes (CPU only), as test_kernel_routes.py asks it."""
import ctypes
import json
import subprocess
import sys

import pytest

import test_kernel_routes as base
from test_lds_limits_step import GRAD, KINDS, LOSS

P, F32, BF16 = base.P, base.F32, base.BF16
RUNS = [(1700, 136, 11000), (900, 8, 33001), (1000, 1536, 32001), (300, 64, 40000), (2305, 264, 9999), (256, 192, 70000)]  # of test_vocab_loss.py's test of these
SINGLE = [(1000, 1544, 32001), (8192, 4096, 131072), (300, 512, 32000), (256, 64, 32000), (16, 1024, 131072)]


def run(runtime):
    """In a process of its own: sizes from standard input, the kernels of a loss and of its gradients (without duplicates) to standard output."""
    hip = ctypes.CDLL(runtime, mode=ctypes.RTLD_GLOBAL)
    lib = ctypes.CDLL(base.LIB)
    lib.lemo_vocab_loss.argtypes, lib.lemo_vocab_loss_grad.argtypes = [KINDS[k] for k in LOSS], [KINDS[k] for k in GRAD]
    seen = ctypes.c_int.in_dll(hip, "n_launched")
    names, blocks = (ctypes.c_char_p * 64).in_dll(hip, "launched"), (ctypes.c_int * 64).in_dll(hip, "blocks")
    out = []
    for dt, M, C, V in json.loads(sys.stdin.read()):
        calls = []
        for call in ((lib.lemo_vocab_loss, (P, M, C, None, M, P, C, C, V, dt, P, 0.0, 0.0, 0.0, P, P, P, P, 1 << 45, None)),
                     (lib.lemo_vocab_loss_grad, (P, 0, P, M, C, None, M, P, C, C, V, dt, P, P, 0.0, 0.0, 0.0, P, C, P, C, 0, P, 1 << 45, None))):
            seen.value = 0
            assert call[0](*call[1]) == 0
            calls.append([[names[i].decode(), blocks[i]] for i in range(seen.value)])
        out.append(calls)
    print(json.dumps(out))


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    folder = tmp_path_factory.mktemp("routes")
    source, runtime = folder / "runtime.c", folder / "runtime.so"
    source.write_text(base.RUNTIME)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", str(source), "-o", str(runtime)], check=True)

    def ask(sizes):
        r = subprocess.run([sys.executable, __file__, str(runtime)], input=json.dumps(sizes), capture_output=True, text=True)
        assert r.returncode == 0, r.stdout + r.stderr
        return json.loads(r.stdout)
    return ask


def test_runs_of_tiles_only_where_they_are_faster(launches):
    runs = [loss[0] for loss, _ in launches([(BF16, *s) for s in RUNS])]
    assert all("vocab_stats_run_kernel" in name and blocks == 256 for name, blocks in runs), runs
    single = [loss[0] for loss, _ in launches([(BF16, *s) for s in SINGLE])]
    assert all("vocab_tile_kernel" in name for name, _ in single), single


def test_few_launches(launches):
    """A loss of few rows: the tiles and one join, which adds the losses too; gradients of one piece: G, dW, dX and its sum."""
    (loss, grad), (many, _), (f32, _) = launches([(BF16, 16, 4096, 32000), (BF16, 17, 4096, 32000), (F32, 16, 1024, 32000)])
    assert len(loss) == 2 and len(many) == 3 and len(f32) == 3 and len(grad) == 4, (loss, many, f32, grad)


def test_gradients_go_by_pieces_of_g(launches):
    """4096 rows, 131072 words: four pieces of 256 MB, three products each, and one sum."""
    (_, grad), = launches([(BF16, 4096, 4096, 131072)])
    assert len(grad) == 13, grad


if __name__ == "__main__":
    run(sys.argv[1])
