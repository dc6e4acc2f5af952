"""As test_lds_limits.py, for the loss over a vocabulary: the first call for a type raises the dynamic-LDS limits of all kernels that its calls may
take.  (The rotation of queries and keys and dropout ask for no dynamic LDS.)"""
import ctypes
import subprocess
import sys

import pytest

import test_lds_limits as base
from test_lds_limits import BF16, F32, FAR, P

KINDS = {"p": ctypes.c_void_p, "i": ctypes.c_int32, "l": ctypes.c_int64, "f": ctypes.c_float, "z": ctypes.c_size_t}
LOSS, GRAD = "pllpl" "pl" "iii" "p" "fff" "ppp" "pzp", "pl" "pllpl" "pl" "iii" "pp" "fff" "plpl" "i" "pzp"
SHAPES = [(1, 8, 1), (1, 4096, 32000), (16, 1024, 131072), (100, 768, 50001), (300, 4096, 131072), (777, 768, 50001), (1500, 256, 1003), (4096, 4096, 131072), (20000, 64, 8192),
          (4096, 256, 131072)]


def loss(lib, dt, _):
    for M, C, V in SHAPES:
        yield lib.lemo_vocab_loss, tuple(KINDS[k](a) for k, a in zip(LOSS, (P, M, C, None, M, P, C, C, V, dt, P, 30.0, 0.1, 0.0, P, P, P, P, 1 << 45, None), strict=True))


def gradient(lib, dt, _):
    for M, C, V in SHAPES:
        for piece in (0, 512):
            for dX, dW in ((FAR, None), (FAR, FAR), (None, FAR)):
                yield lib.lemo_vocab_loss_grad, tuple(KINDS[k](a) for k, a in zip(GRAD, (P, 0, P, M, C, None, M, P, C, C, V, dt, P, P, 0.0, 0.0, 0.0, dX, C, dW, C, piece, P, 1 << 45, None),
                                                                                  strict=True))


ENTRIES = {"loss": (loss, [(F32, 0), (BF16, 0)]), "gradient": (gradient, [(F32, 0), (BF16, 0)])}


@pytest.mark.parametrize("name", list(ENTRIES))
def test_limits_are_raised_in_the_first_call(tmp_path, name):
    source, runtime = tmp_path / "runtime.c", tmp_path / "runtime.so"
    source.write_text(base.RUNTIME)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", str(source), "-o", str(runtime)], check=True)
    r = subprocess.run([sys.executable, __file__, str(runtime), name], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    base.ENTRIES = ENTRIES
    base.run(sys.argv[1], sys.argv[2])
