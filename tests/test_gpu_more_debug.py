"""Rotation, attention with a window and scoring of hidden states through the debug build (bounds checks before the kernels'
stores): no check fails and the results are those of the normal build, bit for bit. In child processes, as a process loads one
of the two libraries."""
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
from paper_2607_07964_gb300.serving import KvCache, Rotation, rotation_theta, score_hidden, score_hidden_grad
g = torch.Generator("cuda").manual_seed(0)
rand = lambda *s: torch.randn(*s, device="cuda", generator=g)
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
digest = lambda t: hashlib.sha256(t.cpu().contiguous().view(torch.uint8).numpy().tobytes()).hexdigest()
res = {}
for T, dim, rot, dtype, pairs in ((1, 128, 128, torch.bfloat16, False), (700, 80, 34, torch.float32, False), (33, 256, 256, torch.float32, True),
                                  (2500, 64, 64, torch.bfloat16, False)):
    theta, scale = rotation_theta(rot, stretch=2.0)
    w = (rand(dim) + 1).to(dtype)
    r = Rotation(theta, scale, pairs, w, w)
    q, k, gq, gk = (rand(T, h, dim).to(dtype) for h in (5, 2, 5, 2))
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 977
    sums = r.grad(q, k, gq, gk, pos=pos)
    r(q, k, pos=pos)
    res[f"rotate {T} {dim}"] = [digest(t) for t in (q, k, gq, gk) + sums]
for heads, dim, group, page, window, sink, dtype in ((2, 128, 4, 64, 100, 4, torch.bfloat16), (3, 64, 5, 16, 33, 20, torch.float32),
                                                     (1, 128, 16, 48, 1, 0, torch.float32)):
    c = KvCache(3, heads, dim, 900, page=page)
    out = []
    for counts in ([600, 1, 77], [1, 1, 1], [0, 40, 2], [90, 0, 0]):
        T, start = sum(counts), i32([0, counts[0], counts[0] + counts[1], sum(counts)])
        c.append(rand(T, heads, dim).to(dtype), rand(T, heads, dim).to(dtype), start, max(counts))
        lse = torch.empty(T, heads * group, device="cuda")
        out += [c.attend(rand(T, heads * group, dim).to(dtype), start, lse=lse, window=window, sink=sink), lse]
    c.check()
    res[f"window {heads} {dim}"] = [digest(t) for t in out]
for T, V, d in ((1, 1, 8), (5, 1001, 72), (90, 5003, 320), (128, 129, 1000), (129, 700, 64), (1000, 3001, 264), (40, 12001, 136), (20, 1000, 2048), (90, 3000, 1032)):
    x, w = rand(T, d).bfloat16(), (rand(V, d) / d ** 0.5).bfloat16()
    y = torch.arange(T, device="cuda") % (V + 1) - 1
    logp, h, lse = score_hidden(x, w, y)
    gx, gw = score_hidden_grad(x, w, y, lse, logp, h, h)
    res[f"linear {T} {V}"] = [digest(t) for t in (logp, h, lse, gx, gw)]
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
