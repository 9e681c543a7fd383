"""Appending without a page table, and first calls of a process inside a stream capture.  Needs an MI355X (-m gpu)."""
import os
import subprocess
import sys

import pytest

from paper_2510_07535_amd import workloads as W
from test_gpu_append import TYPES, Append

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("dtype,quant", TYPES)
def test_append_without_a_page_table(dtype, quant):
    a = Append(21, dtype=dtype, quant=quant, Hq=4, Hkv=2, D=128, ctx=[45], n=37, rot_dim=128)
    a.table = a.dtable = None
    a.run()
    a.check()
    assert int(a.status.item()) == 0


FIRST_CALLS = """
import numpy as np, torch
import block_helpers as H, test_gpu_append as T, test_gpu_logprobs as P
from oracle import cache_blocks as C
from paper_2510_07535_amd import binding as B, workloads as W
def replayed(call):
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        call()
    graph.replay()
    torch.cuda.synchronize()
for quant in (False, True):
    a = T.Append(10, dtype=W.DT_BF16, quant=quant, Hq=8, Hkv=2, D=128, ctx=[90, 33], n=24, rot_dim=128)
    call = B.owl_append_kv_quant if quant else B.owl_append_kv
    replayed(lambda: call(a.desc, a.app, a.dq, a.dk, a.dv, a.freq, None, a.q_out, *a.dev, a.dtable, a.dlens, None, a.status))
    a.check()
bc = H.block_case("first", 6, dtype=W.DT_BF16, Hq=8, Hkv=2, D=128, ctx_lens=[500, 100], trees=[W.chain_tree(8)] * 2)
step = H.QuantStep(bc)
B.owl_verify_attn_quant_init(step.desc)
replayed(step.run)
H.assert_attention(step.result(), bc, H.oracle_out(bc))
acc, na = np.tile(np.array([1, 3] + [-1] * 6, np.int32), (2, 1)), np.array([2, 2], np.int32)
lists = H.i32(acc), H.i32(na)
replayed(lambda: B.owl_commit_kv_quant(step.desc, step.k, step.v, step.ks, step.vs, step.table, step.lens, *lists, None, step.status))
for blocks, raw in ((bc.k, step.k), (bc.v, step.v)):
    blocks.commit(bc.case.page_table, bc.case.ctx_lens, acc, na)
    assert C.same_bytes(raw.cpu().numpy(), blocks.flat)
for rows, vocab in ((3, 1000), (3, 30000), (4, 70001)):
    c = P.Call(H.rng(1).standard_normal((rows, vocab)).astype(np.float32), np.zeros((rows, 1), np.int32), 5)
    replayed(lambda: B.owl_token_logprobs(c.desc, c.x, c.tokens, c.logprob, c.entropy, c.ids, c.top, c.workspace, c.status))
    c.check()
print("all replayed")
"""


def test_first_calls_of_a_process_inside_a_capture():
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([ROOT, os.path.join(ROOT, "tests"), os.environ.get("PYTHONPATH", "")]))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=ROOT, env=env, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "all replayed" in r.stdout, r.stderr[-2000:]
