"""The example decoder's long contexts where each token reads one page."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_lists_of_one_page(cache):
    """Contexts that are one page read it whole (the bound of the example's other tests); of longer ones it is the last page."""
    import decoder
    codes, last, held = decoder.long_contexts(prompts=(decoder.PAGE - 8, 5), steps=3, room=decoder.PAGE, listed=1, cache=cache, tell=lambda *a: None)
    assert held == [decoder.PAGE - 5, 8]
    whole = decoder.Decoder(pages=64, cache=cache)
    for b in range(2):
        n = codes[b].shape[1]
        table, lens = whole.fork(torch.full((1, 8), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), [-1], [0], [n])
        _, exact = whole.step(decoder.columns([codes[b]]), [n], table, torch.tensor([n], dtype=torch.int32, device="cuda"))
        ref, got = exact[:, -1].cpu().double(), last[:, b].double()
        assert (got - ref).norm() <= 0.05 * ref.norm()
    whole.close()
    codes, last, held = decoder.long_contexts(prompts=(150, 60), steps=3, room=96, listed=1, cache=cache, tell=lambda *a: None)
    assert held == [99, 63] and last.isfinite().all() and last.abs().sum() > 0
