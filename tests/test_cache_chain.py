"""Append and attend together, where one hands the other what it makes of unusual inputs."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("out", ["f32", "u8"])
@pytest.mark.parametrize("new", [1, 7, 40, 300])
def test_zero_activations_give_zeros(new, out, cache):
    """A warm-up call: zeros through both operators, norms and rotation included, with columns before their sequence and of none."""
    heads, kv, dim, page, T = 8, 2, 64, 32, new + 9
    pages = -(-new // page) + 2
    kind = torch.bfloat16 if cache == "bf16" else torch.int8
    k, v = (torch.full(s, 7, dtype=kind, device="cuda") for s in ((1, pages, kv, page, dim), (1, pages, kv, dim, page)))
    scales = [torch.full((1, pages, kv, page), float("nan"), device="cuda") for _ in range(2)] if cache == "s8" else []
    c = sp.make_cache(k, v, *scales)
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")     # noqa: E731
    table = torch.stack((torch.arange(pages), torch.full((pages,), -1))).to(torch.int32).cuda()
    table[1, 0], table[0, pages - 1] = pages - 1, -1
    batch = sp.make_batch(ints(0, new, new + 5), ints(new, 3), table)
    w = torch.ones(dim, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    q = torch.full((T, heads, dim), 9.0, dtype=torch.bfloat16, device="cuda")
    sp.spmm_cache_append(c, 0, batch, torch.zeros(((heads + 2 * kv) * dim, T), device="cuda"), T, T, sp.make_append(heads, "f32", 1.0, 0, w, w, 1e-6, sp.make_rope(512, dim).cuda()), q, stream)
    assert (q == 0).all()
    how = sp.make_attend(heads, max(new, 5), dim ** -0.5, True, 0, out, 0.02, 128 if out == "u8" else 0)
    o = torch.full((heads * dim, T), 77, dtype=torch.float32 if out == "f32" else torch.uint8, device="cuda")
    work = torch.empty(sp.spmm_attend_work_bytes(c, 2, T, how), dtype=torch.uint8, device="cuda")
    sp.spmm_cache_attend(c, 0, batch, q, T, how, o, T, work, stream)
    torch.cuda.synchronize()
    assert (o[:, :new + 5] == (0 if out == "f32" else 128)).all() and (o[:, new + 5:] == 77).all()
