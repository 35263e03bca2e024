"""A process whose threads make the library's first calls at once, each on a stream of its own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import threading
import torch
from paper_2006_02924_b200 import binding as b

def inputs(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    ids = torch.randint(0, 500, (700,), generator=g, device="cuda")
    return dict(x=r(700, 1024).bfloat16(), w=r(512, 1024), dy=r(700, 512).bfloat16(), ids=ids, key=torch.tensor([seed], device="cuda"),
                workers=[r(300000) for _ in range(9)], halves=[r(70000).half() for _ in range(64)])

def work(i):
    x8, w8, dy8 = b.adasum_fp8_pack(i["x"]), b.adasum_fp8_pack_weight(i["w"]), b.adasum_fp8_pack(i["dy"])
    y = b.adasum_fp8_linear(x8, w8, 700, 1024, 512)
    dx = b.adasum_fp8_linear_grad(dy8, w8, 700, 1024, 512)
    call = dict(pre_norm="layer", dropout=0.1, seed=i["key"])
    h, z, stats = b.adasum_residual_norm(i["x"], dx, **call)
    gx, gr = b.adasum_residual_norm_grad(i["x"], h, stats, z, dx, **call)
    _, kept = b.adasum_checkpoint_save(i["x"], "gelu")
    dw, db = b.adasum_checkpoint_weight_grad(kept, i["dy"], 1024, want_bias=True)
    table = b.adasum_embedding_grad(gx, i["ids"], 500)
    return [y, dx, h, z, stats[2:], gx, gr, dw, db, table, b.adasum_reduce(i["workers"]), b.adasum_reduce(i["halves"])]

THREADS = 4
jobs = [inputs(n) for n in range(THREADS)]
streams = [torch.cuda.Stream() for _ in range(THREADS)]
torch.cuda.synchronize()
barrier, got = threading.Barrier(THREADS), [None] * THREADS

def thread(n):
    with torch.cuda.stream(streams[n]):
        barrier.wait()
        got[n] = work(jobs[n])
        streams[n].synchronize()

threads = [threading.Thread(target=thread, args=(n,)) for n in range(THREADS)]
for t in threads:
    t.start()
for t in threads:
    t.join()
for job, results in zip(jobs, got):
    assert results is not None
    for k, (first, again) in enumerate(zip(results, work(job))):
        assert torch.equal(first, again), k
torch.cuda.synchronize()
print("same")
"""


@pytest.mark.parametrize("attempt", range(3))
def test_first_calls_from_four_threads(attempt):
    run = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("same"), run.stdout + run.stderr
