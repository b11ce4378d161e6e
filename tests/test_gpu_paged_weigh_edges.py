"""Decode attention that gathers every row's share: weights that are nobody's hold anything and stay as they are, bit for bit."""

import pytest

from test_gpu_paged import Cache, torch_cuda  # noqa: F401
from test_gpu_paged_weigh import _decode, _shares, _weights

pytestmark = pytest.mark.gpu

PATTERNS = (0x7F812345, 0x7FC00001, -0x00400123, 0x7F800000, -0x00800000, 0x7F7FFFFF, 1, -0x80000000)   # of no number, infinities, the largest, the least, -0


@pytest.mark.parametrize("G,D,dtype,page", [(4, 128, "bf16", 16), (1, 64, "bf16", 64), (16, 256, "bf16", 32), (3, 64, "f32", 16), (8, 256, "f32", 128)])
@pytest.mark.parametrize("lengths", [[1], [0, 15, 16, 17, 2, 3], [5, 0, 4097, 30], [2501, 700, 255]], ids=str)
@pytest.mark.parametrize("decay", [1.0, 0.5, 0.0])
def test_weights_that_are_nobodys(torch_cuda, G, D, dtype, page, lengths, decay):  # noqa: F811
    # behind a sequence's last row, whose neighbours are written four at a time, and in pages that no sequence has
    torch = torch_cuda
    c = Cache(torch, G + D + lengths[0], lengths, layers=2, heads=2, group=G, D=D, dtype=dtype, page=page, spare=3).fill()
    q = c.normal((c.n, 2, 2 * G, D))
    old = _weights(c)
    any_bits = torch.tensor(PATTERNS, dtype=torch.int32, device="cuda").repeat(-(-old.numel() // len(PATTERNS)))[: old.numel()].view(old.shape)
    held = torch.zeros(old.shape, dtype=torch.bool, device="cuda")
    for s, n in enumerate(lengths):
        r = torch.arange(n, device="cuda")
        held[:, c.table[s].long()[r // page], :, r % page] = True
    weights = torch.where(held, old.view(torch.int32), any_bits).view(torch.float32)
    was = weights.clone()
    out = _decode(c, q, weights, decay=decay)
    assert torch.equal(out, c.decode(q))
    assert torch.equal(weights.view(torch.int32)[~held], was.view(torch.int32)[~held])
    assert bool(torch.isfinite(weights[held]).all())
    for s, n in enumerate(lengths):
        r = torch.arange(n)
        ids = c.table[s].cpu().long()[r // page]
        for l in range(2):
            for h in range(2):
                share, before = _shares(c, q, s, l, h), old.cpu().double()[l, ids, h, r % page]
                want = torch.where(r < n - 1, decay * before, 0.0) + share
                # as in the test of the shares
                assert bool(((weights.cpu().double()[l, ids, h, r % page] - want).abs() <= 2.0 ** -16 * share + 2.0 ** -23 * want).all())
