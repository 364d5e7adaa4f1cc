"""A plan's first execute uploads tile tables and clears its status word: on a stream that does not wait for the default one, while the
default stream is busy, it gives the bits of later calls."""
import pytest
import torch

import paper_2208_10391_b200 as mom
import workloads as wl
from gpu_util import check_against_oracle
from test_gpu_graph import _setup

pytestmark = pytest.mark.gpu

CASES = [
    ("tiny", lambda: wl.config_tiny(), mom.VARIANT_3XTF32),                                          # copy table of the fused kernel
    ("property_heavy", lambda: wl.config_property_heavy(n=520), mom.VARIANT_3XTF32_FORCE),           # tile tables of the tcgen05 kernel
    ("section4", lambda: wl.config_paper_chain(), mom.VARIANT_3XTF32),                               # status word only
]


@pytest.mark.parametrize("name,eq,variant", CASES, ids=[c[0] for c in CASES])
def test_first_execute_on_a_side_stream(name, eq, variant):
    eq = eq()
    side = torch.cuda.Stream()
    big = torch.empty(1 << 28, device="cuda")
    plan, run, out, (chain, add), keep = _setup(eq, variant)
    torch.cuda.synchronize()
    for _ in range(40):                                   # some milliseconds of ordinary work on the default stream
        big.zero_()
    got = []
    for _ in range(2):
        with torch.cuda.stream(side):
            run(side.cuda_stream)
            got.append(out.clone())
        side.synchronize()
    torch.cuda.synchronize()
    assert plan.device_status() == (0, 0)
    assert torch.equal(got[0], got[1])
    check_against_oracle(eq, got[0].cpu().numpy(), plan, chain, add)
