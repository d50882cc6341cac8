"""Encode beside a prefill worker's attention (colocate.PrefillWork, beside_prefill): both keep their results to the
bit, and the times come back.  In a process with more hardware queues than streams, as the profile runs."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

_BESIDE = """
import json
import torch
from paper_2609_31551_amd import colocate as K, configs as C, eas, synth
p = C.with_layers(C.CLIP_L336, 2)
n = 16
W = synth.make_weights(p, 0)
items = [torch.from_numpy(a).cuda() for a in synth.make_items(p, n, 0)]
enc = eas.Encoder(p, max_tokens=577 * n, max_seqs=n)
wdev = eas.upload_weights(enc.cfg, W)
packed, cu, grid = enc.pack_microbatch(items)
out = torch.empty((577 * n, p["out_dim"]), dtype=torch.float32, device="cuda")
def run(stream):
    enc.encode_microbatch(packed, cu, grid, wdev, out=out, stream=stream)
work = K.PrefillWork(lens=(130, 577, 64, 900))
torch.cuda.synchronize()
run(torch.cuda.current_stream())
work.step()
torch.cuda.synchronize()
want = [t.clone() for t in (out, work.out, work.out1)]
for t in (out, work.out, work.out1):
    t.zero_()
ms = K.beside_prefill(run, work, reps=2)
torch.cuda.synchronize()
print(json.dumps({"ms": ms, "same": [bool(torch.equal(a, b)) for a, b in zip((out, work.out, work.out1), want)]}))
"""


def test_encode_and_prefill_side_by_side_keep_their_results():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, GPU_MAX_HW_QUEUES="16", PYTHONPATH=root)
    r = subprocess.run([sys.executable, "-c", _BESIDE], env=env, cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    res = json.loads([line for line in r.stdout.splitlines() if line.startswith("{")][-1])
    print("[colocate] CLIP x16, 2 layers, beside prompt and cache attention: %s" % res["ms"], flush=True)
    assert res["same"] == [True, True, True]
    assert set(res["ms"]) == {"encode_alone", "encode_beside", "prefill_alone", "prefill_beside"}
    assert all(v > 0 for v in res["ms"].values())
