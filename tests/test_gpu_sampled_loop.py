"""The decode loop that draws its tokens, whatever torch's default type is."""
import pytest
import torch

from helpers import to_cuda
from paper_2404_08698_amd import binding as B
from paper_2404_08698_amd import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [synth.TINY, synth.MID_GQA], ids=["f32", "mid"])
def test_the_loop_that_draws_under_another_default_type(shape):
    model = B.Model(shape, to_cuda(synth.make_weights(shape, 3)), max_window=16, max_positions=512)
    prompt = synth.workload_prompt("tiny")[:40]

    def run():
        return B.anpd_generate(model, B.KVCache(model, 512), B.NgramTable(2, 4, model.vocab), prompt, 4, 20, sampling=B.SamplingRules(top_p=0.9),
                               generator=torch.Generator(device="cuda").manual_seed(5))["tokens"]

    want = run()
    try:
        for dtype in (torch.float64, torch.bfloat16):
            torch.set_default_dtype(dtype)
            assert run() == want
    finally:
        torch.set_default_dtype(torch.float32)
