"""Runs calls of the library without a GPU: a child process loads tests/host_runtime.cpp in front of the HIP runtime, and
every launch that the library makes is recorded instead of run."""
import atexit
import functools
import json
import os
import shutil
import subprocess
import sys
import tempfile
import textwrap

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@functools.lru_cache(None)
def _library() -> str:
    folder = tempfile.mkdtemp(prefix="kvr_host_runtime_")
    atexit.register(shutil.rmtree, folder, ignore_errors=True)
    out = os.path.join(folder, "libhost_runtime.so")
    src = os.path.join(ROOT, "tests", "host_runtime.cpp")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", src, "-o", out, "-ldl"], check=True, timeout=100)
    return out


PRELUDE = """
import ctypes, json, sys
sys.modules["torch"] = None  # (the library is loaded without it, and it would take seconds)
host = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
host.host_log.restype = ctypes.c_char_p
import paper_2609_17983_amd as kvr

def dims(layers=1, Hq=32, Hkv=8, hd=128, max_ctx=4096, max_rows=64, dtype=kvr.KVR_BF16, d_model=64, vocab=64):
    return kvr.kvr_dims(layers, d_model, Hq, Hkv, hd, 64, vocab, 0, 1e-5, 1e4, max_ctx, max_rows, dtype)

memory = ctypes.create_string_buffer(1 << 22)
P = (ctypes.addressof(memory) + 255) // 256 * 256  # no kernel runs: every device pointer may be this one

def context(d):
    lw = dict.fromkeys(("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down"), P)
    layers = (kvr.kvr_layer_weights * d.n_layers)()
    for l in layers:
        for k, v in lw.items():
            setattr(l, k, v)
    w = kvr.kvr_weights(P, P, layers, P)
    return kvr.kvr_create(d, w)

def launched():
    out = []
    for line in host.host_log().decode().splitlines():
        name, *n = line.split("\\t")
        n = [int(x) for x in n]
        name = name.replace("(anonymous namespace)::", "").replace("kvr::", "").removeprefix("void ").split("(")[0]
        out.append(dict(name=name, grid=n[:3], threads=n[3], lds=n[6]) if n else dict(name=name))
    host.host_clear()
    return out

def attend(ctx, bits, docs):
    # docs: (n_cap, positions)
    lst = kvr.make_packed_rows([(P, n, p) for n, p in docs])
    host.host_clear()
    kvr.kvr_attention_packed(ctx, 0, bits, lst, P, 1 << 16, P, 1 << 16, None)
    return launched()

result = None
"""


def run(body: str):
    """The value that `body`, a script that follows PRELUDE, leaves in `result`."""
    code = PRELUDE + textwrap.dedent(body) + "\nprint('RESULT' + json.dumps(result))\n"
    r = subprocess.run([sys.executable, "-c", code, _library()], cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr
    return json.loads(r.stdout.rsplit("RESULT", 1)[1])
