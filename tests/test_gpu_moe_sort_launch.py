"""The routing table's launch: its shared memory grows with the number of experts (33 words each and a little that is static), so
around 372 experts it passes the 48 KB that a kernel has without asking. A call must not depend on what was called before it, nor on
what another host thread calls meanwhile."""
import subprocess
import sys
import threading
from pathlib import Path

import numpy as np
import pytest
import torch

from paper_2609_39223_b200 import api
from test_gpu_moe import check_table, draw_ids

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent

FIRST_CALL = """
import sys
import torch
from paper_2609_39223_b200 import api
G = int(sys.argv[1])
ids = (7 * torch.arange(30, dtype=torch.int32, device="cuda")).view(15, 2)          # 30 experts with one pair each
plan = api.qf_moe_sort(ids, G)
assert torch.equal(plan.row_of.view(-1).cpu(), 128 * torch.arange(30, dtype=torch.int32))
want = torch.zeros(G, dtype=torch.int32)
want[:210:7] = 1
assert torch.equal(plan.counts.cpu(), want) and plan.group_offsets[-1].item() == 30 * 128
"""


@pytest.mark.parametrize("G", [371, 372, 373, 1024])
def test_first_call_of_a_process(G):
    r = subprocess.run([sys.executable, "-c", FIRST_CALL, str(G)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("T", [40, 5000, 40000])
@pytest.mark.parametrize("G", [371, 372, 373, 1023, 1024])
def test_sort_of_many_experts(T, G):
    """One CTA, a cluster of some and one of 16."""
    ids = draw_ids(np.random.default_rng(T + G), T, 2, G, "even")
    check_table(ids, api.qf_moe_sort(torch.tensor(ids, device="cuda"), G), G)


def test_host_threads_with_different_numbers_of_experts():
    """The C calls run outside the interpreter's lock, so that one thread is between its steps while another begins."""
    tokens, k, calls = 64, 2, 20000
    table = {G: draw_ids(np.random.default_rng(G), tokens, k, G, "even") for G in (380, 700, 1024)}
    failed, plans = [], {}
    go = threading.Barrier(len(table))

    def work(G):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ids = torch.tensor(table[G], device="cuda")
            plan = plans[G] = api.qf_moe_sort(ids, G)
        f = api.lib().qf_moe_sort
        args = (ids.data_ptr(), api.DT_I64, tokens, k, G, plan.rows_padded, plan.row_of.data_ptr(), plan.group_offsets.data_ptr(),
                plan.counts.data_ptr(), stream.cuda_stream)
        go.wait()
        failed.extend((G, code) for code in {f(*args) for _ in range(calls)} if code)
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(G,)) for G in table]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, [(G, api.status_string(code)) for G, code in failed]
    assert len(plans) == len(table)
    for G, plan in plans.items():
        check_table(table[G], plan, G)
