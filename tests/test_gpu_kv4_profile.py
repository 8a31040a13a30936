"""The profile of a forward on the 4-bit cache books every launch of its attention: the kernel, the join of the splits that a long page table allows, the weighing."""
import pytest
import torch

import s2d2_inputs as I
from paper_2603_25702_amd import Params
from paper_2603_25702_amd.runner import Session
from tests.test_gpu_parity import TINY

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("room,budget,draft,verify", [(512, None, 1, 1), (4096, None, 2, 2), (512, 64, 1, 2), (4096, 64, 2, 3)])
def test_attention_launches_of_a_forward(room, budget, draft, verify):
    ses = Session(TINY, I.gen_weights(TINY, 3), 1, 4, room, cache_bits=4, budget=budget)
    ses.prefill([I.gen_prefix_ids(TINY, 100, 3, 0)])
    prm, e = Params(seed=1), ses.eng
    for call, want in ((lambda: e.s2d2_draft(ses.kv, ses.st, 1, 4, prm, ses.d), draft), (lambda: e.s2d2_verify(ses.kv, ses.st, 1, 4, prm, ses.d, ses.v), verify)):
        e.s2d2_profile_start(256)
        call()
        torch.cuda.synchronize()
        assert e.s2d2_profile_stop()["attention"]["launches"] == want * TINY.n_layers
