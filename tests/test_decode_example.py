"""The decoder layer on the paged cache (decode_example.py) beyond the steps that its own run takes.  Needs an MI355X (-m gpu)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_requests_without_a_new_token():
    """Their rows are 0, whichever request comes before them or none; their caches stay, and go on when they have a token again.  The tolerance is that of the example's own
    run: a few roundings of bf16, 2^-8 of the largest output each."""
    from paper_2002_12798_amd import decode_example
    g = torch.Generator().manual_seed(8)
    layer = decode_example.PagedAttention(256, 4, 2, 64, 4, 60)
    history = [torch.empty((0, 256), device="cuda") for _ in range(4)]
    for fresh in ([0, 12, 0, 1], [1, 0, 30, 0], [0, 0, 0, 1], [2, 1, 0, 0], [1, 1, 1, 1]):
        x = torch.randn((sum(fresh), 256), generator=g).bfloat16().cuda()
        y = layer.step(x, torch.tensor(fresh, dtype=torch.int32, device="cuda")).float()
        for r, part in enumerate(x.split(fresh)):
            history[r] = torch.cat([history[r], part.float()])
            if not fresh[r]:
                assert (y[r] == 0).all()
                continue
            want = layer.plain(history[r])
            assert (y[r] - want).abs().max() < 8 * 2.0 ** -8 * want.abs().max()
