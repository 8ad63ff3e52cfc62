"""Runs calls of the operators around the layer against the stand-in HIP runtime (_fake_hip.c) in a process of its own and reports their kernel launches:
`python -m tests._fake_hip_layer stand_in.so < calls.json`.  A call is {"entry": "linear", M, N, K, "exact"} or {"entry": "attention", T, heads, kv_heads, dim,
"page", "max_pages", "e4m3", "heads_first", "window"}.  Not collected by pytest."""
import ctypes as C
import json
import os
import re
import subprocess
import sys
import types

HERE = os.path.dirname(os.path.abspath(__file__))


def trace(calls, tmp_path):
    """[{status, launches: [{name, args (the template's, as numbers), grid, block, lds}]}] of the calls, from a fresh process."""
    so = os.path.join(str(tmp_path), "fake_hip.so")
    if not os.path.exists(so):
        subprocess.run(["gcc", "-O1", "-shared", "-fPIC", os.path.join(HERE, "_fake_hip.c"), "-o", so], check=True)
    r = subprocess.run([sys.executable, "-m", "tests._fake_hip_layer", so], input=json.dumps(calls), capture_output=True, text=True,
                       cwd=os.path.dirname(HERE), timeout=120)
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


class _Torch(types.ModuleType):
    def __getattr__(self, name):                   # dtypes and the like: never used here
        return object()


def _main():
    stub = _Torch("torch")                          # torch brings the real HIP runtime into the process
    stub.Tensor = object
    stub._C = types.SimpleNamespace(_cuda_getCurrentRawStream=None)
    sys.modules["torch"] = stub
    from tests._fake_hip import _Dim3
    fake = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
    package = types.ModuleType("paper_2507_17133_amd")
    package.__path__ = [os.path.join(os.path.dirname(HERE), "paper_2507_17133_amd")]
    sys.modules["paper_2507_17133_amd"] = package
    from paper_2507_17133_amd import layer as L
    lib, launches = L._lib(), []

    def on_launch(name, grid, block, lds, args):
        name = name.decode()
        m = re.match(r"_ZN4bmoe(?:12_GLOBAL__N_1)?(\d+)", name)
        plain = name[m.end():m.end() + int(m.group(1))] if m else name
        numbers = re.match(r"I((?:L[ib]\d+E)+)E", name[m.end() + len(plain):]) if m else None
        launches.append({"name": plain, "args": [int(v) for v in re.findall(r"L[ib](\d+)E", numbers.group(1))] if numbers else [],
                         "grid": [grid.x, grid.y, grid.z], "block": block.x, "lds": lds})
        return 0

    cb = C.CFUNCTYPE(C.c_int, C.c_char_p, _Dim3, _Dim3, C.c_size_t, C.POINTER(C.c_void_p))(on_launch)
    fake.fake_on_launch(cb)
    p = lambda i: 0x1000000000 * (i + 1)            # never read or written
    out = []
    for c in json.load(sys.stdin):
        launches.clear()
        if c["entry"] == "linear":
            M, N, K = c["M"], c["N"], c["K"]
            a = L.moe_linear_args(x8=p(0), x_stride=K, x_scale=p(1), x_scale_stride=max(M, 1), w8=p(2), w_scale=p(3), out=p(4), out_stride=N, M=M, N=N, K=K,
                                  exact=c.get("exact", 0))
            st = lib.moe_linear_e4m3(C.byref(a), p(5), 1 << 45, None)
        elif c["entry"] == "attention":
            D, Hk, page, hf = c["dim"], c["kv_heads"], c["page"], c.get("heads_first", False)
            cache = L.moe_kv_cache(k=p(0), v=p(1), page_stride=page * Hk * D, token_stride=D if hf else Hk * D, head_stride=page * D if hf else D, k_scale=p(2),
                                   v_scale=p(3), type=1 if c.get("e4m3") else 0, n_pages=c.get("n_pages", 1000), page_size=page, n_kv_heads=Hk, head_dim=D)
            T, H = c["T"], c["heads"]
            table = L.moe_block_table(pages=p(4), row_stride=c["max_pages"], token_row=None, n_rows=T, max_pages=c["max_pages"])
            st = lib.moe_paged_attention(C.byref(cache), C.byref(table), p(5), H * D, H, T, p(6), 0.1, c.get("window", 0), p(7), H * D, None, p(8), 1 << 40, None)
        else:
            raise ValueError(c["entry"])
        out.append({"status": st, "launches": list(launches)})
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main()
