"""The paged read on another stream than the current one (needs a GB300)."""
import pytest
import torch

from paper_2602_07160_gb300 import fem
from tests.test_gpu_paged_read import lib, make, make_beta  # noqa: F401  (lib: builds and loads the library)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 40])
def test_outputs_on_another_stream_are_their_own_memory(n):
    """A tensor of the outputs' size, released while the current stream has still to write it, is not what a
    call on another stream returns."""
    q, cache, off, ctx, table = make("bf16", 2, 4, 128, 64, [(n, 500)], seed=60)
    beta = make_beta((0.1, 5.0), 2, 128)
    want, want_lse = fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=n)
    want_k, want_v = fem.fem_cache_gather(cache, table, ctx * 0, torch.tensor([0, 500], dtype=torch.int32, device="cuda"), 500)
    offsets, starts = torch.tensor([0, 500], dtype=torch.int32, device="cuda"), ctx * 0
    side = torch.cuda.Stream()
    late = [torch.empty_like(t) for t in (want, want_lse, want_k, want_v)]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)  # some ten milliseconds
    for t in late:
        t.fill_(7)
    del late, t
    out, lse = fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=n, stream=side)
    k, v = fem.fem_cache_gather(cache, table, starts, offsets, 500, stream=side)
    torch.cuda.synchronize()
    fem.check_device_error()
    for got, wanted in ((out, want), (lse, want_lse), (k, want_k), (v, want_v)):
        assert torch.equal(got, wanted)
