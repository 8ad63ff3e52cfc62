"""Runs calls of the operators of a step with several new tokens against the stand-in HIP runtime (_fake_hip.c) in a process of its own and reports their
kernel launches: `python -m tests._fake_hip_draft stand_in.so < calls.json`.  A call is {"entry": "logprob", T, V, fp32, given, top, stride, "off"} or
{"entry": "chunk", T, seqs, heads, kv_heads, dim, page, max_pages, e4m3, tree}.  Not collected by pytest."""
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
    r = subprocess.run([sys.executable, "-m", "tests._fake_hip_draft", so], input=json.dumps(calls), capture_output=True, text=True,
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
    from paper_2507_17133_amd import draft as M
    lib, launches = M._lib(), []

    def on_launch(name, grid, block, lds, args):
        name = name.decode()
        m = re.search(r"(slice_kernel|join_rows|chunk_kernel|chunk_join|move_kernel)", name)
        launches.append({"name": m.group(1) if m else name, "args": [int(v) for v in re.findall(r"L[ib](\d+)E", name)], "grid": [grid.x, grid.y, grid.z],
                         "block": block.x, "lds": lds})
        return 0

    cb = C.CFUNCTYPE(C.c_int, C.c_char_p, _Dim3, _Dim3, C.c_size_t, C.POINTER(C.c_void_p))(on_launch)
    fake.fake_on_launch(cb)
    p = lambda i: 0x1000000000 * (i + 1)            # never read or written
    out = []
    for c in json.load(sys.stdin):
        launches.clear()
        if c["entry"] == "logprob":
            T, V, G, N = c["T"], c["V"], c.get("given", 0), c.get("top", 0)
            a = M.moe_logprob_args(logits=p(0) + c.get("off", 0), stride=c.get("stride", V), tokens=p(1) if G else None, tokens_stride=G, logprob=p(2) if G else None,
                                   rank=p(3) if G else None, lse=p(4), entropy=p(5), top_id=p(6) if N else None, top_logprob=p(7) if N else None, T=T, V=V,
                                   type=1 if c.get("fp32") else 0, n_given=G, n_top=N)
            st = lib.moe_token_logprobs(C.byref(a), p(8), 1 << 45, None)
        elif c["entry"] == "chunk":
            D, Hk, page = c["dim"], c["kv_heads"], c["page"]
            cache = M.moe_kv_cache(k=p(0), v=p(1), page_stride=page * Hk * D, token_stride=Hk * D, head_stride=D, k_scale=p(2), v_scale=p(3),
                                   type=1 if c.get("e4m3") else 0, n_pages=c.get("n_pages", 1000), page_size=page, n_kv_heads=Hk, head_dim=D)
            T, H, B = c["T"], c["heads"], c["seqs"]
            table = M.moe_block_table(pages=p(4), row_stride=c["max_pages"], token_row=None, n_rows=B, max_pages=c["max_pages"])
            tree = c.get("tree", False)
            ch = M.moe_chunk(first=p(5), context=p(6), seen=p(7) if tree else None, seen_stride=2, positions=None, seen_words=2 if tree else 0, n_seqs=B, T=T,
                             window=0, sinks=0)
            st = lib.moe_chunk_attention(C.byref(cache), C.byref(table), C.byref(ch), p(8), H * D, H, 0.1, p(9), H * D, None, p(10), 1 << 40, None)
        else:
            raise ValueError(c["entry"])
        out.append({"status": st, "launches": list(launches)})
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main()
