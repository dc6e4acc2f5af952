"""As test_lds_limits.py, for the attention over chosen key blocks: the first call of an entry point for a type and head size raises the
dynamic-LDS limits of all kernels that its calls may take."""
import ctypes
import subprocess
import sys

import pytest

import test_lds_limits as base
from test_lds_limits import BF16, F32, FAR, P

KINDS = {"p": ctypes.c_void_p, "i": ctypes.c_int32, "l": ctypes.c_int64, "f": ctypes.c_float, "z": ctypes.c_size_t}
TYPES = {"select_blocks": "pliiiillpllii" "iipp", "select_blocks_step": "piiiiillplpiipp", "block_attention": "pppll" "iiii" "llllll" "piiilfi" "pllppzp",
         "block_attention_grad": "pppppp" "ll" "iiii" "llllllllll" "piiilfi" "pppp" "zp", "block_attention_step": "pppil" "iiii" "ll" "llllll" "ppii" "f" "pllpzp"}


def typed(lib, name, *args):
    return getattr(lib, "lemo_" + name), tuple(KINDS[k](a) for k, a in zip(TYPES[name], args, strict=True))


# queries, keys, heads, key heads, block of keys, of queries, blocks listed
LISTS = [(1, 1, 1, 1, 32, 1, 1), (32768, 32768, 32, 8, 64, 64, 16), (8192, 8192, 32, 16, 64, 64, 16), (8192, 8192, 32, 32, 64, 64, 16), (2999, 2999, 32, 8, 64, 16, 12),
         (1000, 1000, 16, 4, 32, 1, 8), (3001, 3001, 16, 16, 32, 1, 12), (300, 300, 8, 8, 32, 1, 9), (64, 900000, 4, 4, 64, 64, 1900), (2, 500000, 4, 4, 32, 1, 3840),
         (5000, 5000, 16, 1, 128, 1, 4), (700, 524288, 2, 2, 32, 64, 64), (4000, 524288, 4, 4, 32, 1, 64)]


def select(lib, dt, d):
    for S_q, S_k, H, H_kv, b, bq, T in LISTS:
        yield typed(lib, "select_blocks", P, S_q, H, H_kv, d, dt, H * d, d, P, S_k, 0, b, bq, T, 0, FAR, None)


def select_step(lib, dt, d):
    for B, S, H, H_kv, T in [(1, 100, 1, 1, 1), (1, 32768, 32, 8, 16), (64, 16384, 32, 8, 16), (2000, 16384, 32, 8, 16), (3, 524288, 8, 8, 100)]:
        yield typed(lib, "select_blocks_step", P, B, H, H_kv, d, dt, H * d, d, P, S, P, 32, T, FAR, None)


def attention(lib, dt, d):
    for S_q, S_k, H, H_kv, b, bq, T in LISTS:
        for flags in (1, 0):
            yield typed(lib, "block_attention", P, P, P, S_q, S_k, H, H_kv, d, dt, H * d, d, H_kv * d, d, H_kv * d, d, P, T, b, bq, 0, 0., flags, FAR, H * d, d, P, P,
                                             1 << 40, None)


def attention_step(lib, dt, d):
    for B, S, H, H_kv, T in [(1, 100, 1, 1, 1), (1, 32768, 32, 8, 16), (64, 16384, 32, 8, 16), (2000, 16384, 32, 8, 16), (3, 524288, 512, 1, 100)]:
        yield typed(lib, "block_attention_step", P, P, P, B, S, H, H_kv, d, dt, H * d, d, S * H_kv * d, H_kv * d, d, S * H_kv * d, H_kv * d, d, P, P, T, 64, 0., FAR, H * d, d,
                                              P, 1 << 40, None)


def gradient(lib, dt, d):
    for S_q, S_k, H, H_kv, b, bq, T in LISTS:
        if S_k <= 16384 * b:
            yield typed(lib, "block_attention_grad", P, P, P, P, P, P, S_q, S_k, H, H_kv, d, dt, H * d, d, H * d, d, H_kv * d, d, H_kv * d, d, H * d, d,
                        P, T, b, bq, 0, 0., 1, FAR, FAR, FAR, P, 1 << 40, None)


ENTRIES = {"select": (select, [(dt, d) for dt in (F32, BF16) for d in (64, 128)]), "select_step": (select_step, [(dt, d) for dt in (F32, BF16) for d in (64, 128)]),
           "attention": (attention, [(BF16, 64), (BF16, 128)]), "attention_step": (attention_step, [(BF16, 64), (BF16, 128)]),
           "gradient": (gradient, [(BF16, 64), (BF16, 128)])}


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
