"""The example decoder: prompts in chunks, beams that fork, pages that are moved -- and the same sequences in one piece each."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_beams_attend_to_what_a_whole_prompt_does(cache):
    """The codes between layers are rounded twice on the way (weights to 16 bits by another kernel, results to 8 bits), so that a
    code may differ by one; the last layer's attention is compared where it comes from: a few parts in a hundred of its size."""
    import decoder
    codes, last, used = decoder.main(cache=cache, tell=lambda *a: None)
    assert used[0] == 0 and 0 < used[2] <= 64
    whole = decoder.Decoder(pages=64, cache=cache)
    for b in (0, 3, 5, 7):
        n = codes[b].shape[1]
        table, lens = whole.fork(torch.full((1, 8), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), [-1], [0], [n])
        _, exact = whole.step(decoder.columns([codes[b]]), [n], table, torch.tensor([n], dtype=torch.int32, device="cuda"))
        ref, got = exact[:, -1].cpu().double(), last[:, b].double()
        assert (got - ref).norm() <= 0.05 * ref.norm()
    whole.close()
