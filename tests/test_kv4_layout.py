"""The 4-bit cache's layout: every code has a place of its own, and the places fill the codes' bytes."""
import pytest
import torch

from tests import kv4_common as Q


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 1024])
def test_places_are_one_to_one(page, dim):
    for byte, shift in Q.places(page, dim):
        at = (2 * byte + shift // 4).flatten().sort().values
        assert torch.equal(at, torch.arange(page * dim))


@pytest.mark.parametrize("dim", [64, 128])
def test_a_token_has_whole_bytes_of_its_own(dim):
    for byte, _ in Q.places(64, dim):
        owners = [set(row.tolist()) for row in byte]
        assert all(len(o) == dim // 2 for o in owners) and len(set.union(*owners)) == 64 * dim // 2


def test_reading_back_what_was_written():
    page, dim = 16, 64
    cache = torch.zeros((1, 1, 2, Q.part_bytes(page, dim)), dtype=torch.uint8)
    u = torch.randint(0, 16, (2, page, dim), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    for which, (byte, shift) in enumerate(Q.places(page, dim)):
        for t in range(page):
            for d in range(dim):
                cache[0, 0, which, byte[t, d]] |= int(u[which, t, d]) << int(shift[t, d])
        cache[0, 0, which, page * dim // 2:] = torch.full((page * dim // 32,), 0.5, dtype=torch.float16).view(torch.uint8)
    for which, (codes, scales) in enumerate(Q.read(cache, page, dim)):
        assert torch.equal(codes[0, 0], u[which]) and (scales == 0.5).all()
