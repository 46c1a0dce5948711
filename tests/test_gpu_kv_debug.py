"""Decoding and scoring through the debug build (bounds checks before the kernels' stores): no check fails
and the results are those of the normal build, bit for bit. In child processes, as a process loads
one of the two libraries."""
import json
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import hashlib, json, os, sys
import torch
sys.path.insert(0, os.environ["KQ_ROOT"])
from paper_2607_07964_gb300 import kronq as K
from paper_2607_07964_gb300.serving import KvCache
g = torch.Generator("cuda").manual_seed(0)
rand = lambda *s: torch.randn(*s, device="cuda", generator=g)
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
digest = lambda t: hashlib.sha256(t.cpu().contiguous().view(torch.uint8).numpy().tobytes()).hexdigest()
res = {}
for name, heads, dim, group, page, dtype in (("a", 2, 128, 4, 64, torch.bfloat16), ("b", 3, 64, 5, 16, torch.float32),
                                             ("c", 1, 128, 16, 48, torch.float32)):
    c = KvCache(3, heads, dim, 700, page=page, budget=300, recent=40, sink=3)
    out = []
    for counts in ([600, 1, 77], [1, 1, 1], [0, 40, 2], [1, 1, 0], [90, 0, 0], [1, 1, 1]):
        T, start = sum(counts), i32([0, counts[0], counts[0] + counts[1], sum(counts)])
        c.append(rand(T, heads, dim).to(dtype), rand(T, heads, dim).to(dtype), start, max(counts))
        out.append(digest(c.attend(rand(T, heads * group, dim).to(dtype), start)))
    c.check()
    k, v = c.read(dtype)
    n = int(c.lens.min())
    res[name] = out + [digest(t) for t in (k, v, c.lens, c.seen, c.acc[..., :n], c.pos[..., :n])]
for V, dtype in ((5003, torch.bfloat16), (40001, torch.float32), (100, torch.bfloat16)):
    x, y = rand(9, V).to(dtype), torch.arange(9, device="cuda")
    logp, h, lse, tl = torch.empty(9, device="cuda"), torch.empty(9, device="cuda"), torch.empty(9, device="cuda"), torch.empty(9, 7, device="cuda")
    ids = torch.empty(9, 7, dtype=torch.int32, device="cuda")
    K.kq_token_logprobs(x, y, logp, entropy=h, lse=lse, top_id=ids, top_logp=tl)
    grad = torch.empty_like(x)
    K.kq_token_logprobs_grad(x, y, lse, logp, grad, entropy=h, g_entropy=h)
    res[str(V)] = [digest(t) for t in (logp, h, lse, ids, tl, grad)]
print(json.dumps({"debug": K.kq_debug_build(), "res": res, "after": K.kq_debug_status()}))
'''


def _child(debug: bool) -> dict:
    env = dict(os.environ, KQ_ROOT=ROOT, KQ_DEBUG="1" if debug else "0")
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


def test_debug_build_finds_no_store_out_of_bounds_and_agrees():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_07964_gb300 import build
    build.build()
    build.build(debug=True)
    dbg, rel = _child(True), _child(False)
    assert dbg["debug"] == 1 and rel["debug"] == 0
    assert dbg["after"] == [None, 0], dbg["after"]
    assert dbg["res"] == rel["res"]
