"""Runs moe_token_logprobs against the stand-in HIP runtime (_fake_hip.c) in a process of its own and reports which rows of its arguments each launch takes:
`python -m tests._fake_hip_rows stand_in.so < calls.json`.  A call is {T, V, fp32, given, top, stride}.  Not collected by pytest."""
import ctypes as C
import json
import os
import subprocess
import sys
import types

from tests._fake_hip_draft import HERE, _Torch

POINTERS = ("logits", "tokens", "logprob", "rank", "lse", "entropy", "top_id", "top_logprob")


class _Args(C.Structure):                              # what the kernels get, in the order of LogprobArgs
    _fields_ = [("logits", C.c_uint64), ("stride", C.c_int64), ("tokens", C.c_uint64), ("tokens_stride", C.c_int64)] + [(n, C.c_uint64) for n in POINTERS[2:]] + [
        (n, C.c_int32) for n in ("T", "V", "G", "N", "slices")]


def trace(calls, tmp_path):
    """[{status, base: {pointer of the call}, launches: [{name, T, pointers}]}]"""
    so = os.path.join(str(tmp_path), "fake_hip.so")
    if not os.path.exists(so):
        subprocess.run(["gcc", "-O1", "-shared", "-fPIC", os.path.join(HERE, "_fake_hip.c"), "-o", so], check=True)
    r = subprocess.run([sys.executable, "-m", "tests._fake_hip_rows", so], input=json.dumps(calls), capture_output=True, text=True, cwd=os.path.dirname(HERE), timeout=120)
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


def _main():
    stub = _Torch("torch")                              # torch brings the real HIP runtime into the process
    stub.Tensor = object
    stub._C = types.SimpleNamespace(_cuda_getCurrentRawStream=None)
    sys.modules["torch"] = stub
    from tests._fake_hip import _Dim3
    fake = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
    package = types.ModuleType("paper_2507_17133_amd")
    package.__path__ = [os.path.join(os.path.dirname(HERE), "paper_2507_17133_amd")]
    sys.modules["paper_2507_17133_amd"] = package
    from paper_2507_17133_amd import draft as M
    lib, launches = M._lib(), []

    def on_launch(name, grid, block, lds, args):
        a = C.cast(args[0], C.POINTER(_Args))[0]
        launches.append(dict({"name": "join" if b"join_rows" in name else "slice", "T": a.T}, **{n: getattr(a, n) for n in POINTERS}))
        return 0

    cb = C.CFUNCTYPE(C.c_int, C.c_char_p, _Dim3, _Dim3, C.c_size_t, C.POINTER(C.c_void_p))(on_launch)
    fake.fake_on_launch(cb)
    out = []
    for c in json.load(sys.stdin):
        launches.clear()
        G, N = c["given"], c["top"]
        base = {n: (i + 1) << 44 for i, n in enumerate(POINTERS)}       # never read or written
        if not G:
            base.update(tokens=0, logprob=0, rank=0)
        if not N:
            base.update(top_id=0, top_logprob=0)
        a = M.moe_logprob_args(stride=c["stride"], tokens_stride=G + 2, T=c["T"], V=c["V"], type=1 if c["fp32"] else 0, n_given=G, n_top=N, **{k: v or None for k, v in base.items()})
        st = lib.moe_token_logprobs(C.byref(a), 1 << 50, 1 << 60, None)
        out.append({"status": st, "base": base, "launches": list(launches)})
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main()
