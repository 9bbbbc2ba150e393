"""What calls of the library would launch, without a GPU and without torch: run as a program, in a process whose LD_PRELOAD names the
recorder made of launch_sizes.c, it makes the calls that it reads and prints what they answer and launch; `record` is for tests.

A call is [function, [[kind, value], ...]], kind one of i (int), u (unsigned), f (float), z (size_t), p (address), rows ([address, row]) and heads
([address, token, head]); values of None are NULL.
"""
import ctypes
import json
import os
import struct
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))


def make_recorder(folder):
    so = os.path.join(str(folder), "launch_sizes.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "launch_sizes.c")], check=True)
    return so


def record(recorder, path, calls):
    """[(status, [(kernel, grid, block), ...]), ...] of the calls."""
    env = dict(os.environ)
    env["LD_PRELOAD"] = recorder + (":" + env["LD_PRELOAD"] if env.get("LD_PRELOAD") else "")
    r = subprocess.run([sys.executable, os.path.abspath(__file__), path, recorder], input=json.dumps(calls), env=env, capture_output=True, text=True,
                       timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    return [(status, [(line.split()[0], *(tuple(map(int, line.split()[i:i + 3])) for i in (1, 4))) for line in launched]) for status, launched in json.loads(r.stdout)]


def _argument(kind, value):
    if kind == "p" or value is None:
        return ctypes.c_void_p(value)
    if kind in ("rows", "heads"):
        return struct.pack("Pq" if kind == "rows" else "Pqq", *value)
    return {"i": ctypes.c_int, "u": ctypes.c_uint, "f": ctypes.c_float, "z": ctypes.c_size_t}[kind](value)


def _main(path, recorder):
    rec, L, out = ctypes.CDLL(recorder), ctypes.CDLL(path), []
    rec.recorded_launches.restype = ctypes.c_char_p
    for name, args in json.load(sys.stdin):
        rec.recorded_launches()
        status = getattr(L, name)(*(_argument(*a) for a in args))
        out.append([status, rec.recorded_launches().decode().splitlines()])
    print(json.dumps(out))


if __name__ == "__main__":
    _main(*sys.argv[1:])
