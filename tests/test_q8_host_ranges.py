"""What the operators round a cache in 8 bits take and refuse at the ends of their ranges: nothing here needs a GPU."""
import torch

from paper_2511_08003_b200 import binding as sv


def test_one_token_in_a_plane_with_heads_far_apart():
    """A single token needs no token stride: none may come of a head stride that would be refused as one (2 GB)."""
    cache = torch.empty((8, 1 << 20, 128), dtype=torch.bfloat16, device="meta")
    for n in (1, 2, 9):
        address, token, head = sv._token_rows(cache[:, 7:7 + n].transpose(0, 1), n, 8, 128)
        assert (token, head) == (128, 128 << 20)
    assert sv._token_rows(cache[:1, 7:8].transpose(0, 1), 1, 1, 128)[1:] == (128, 128)
    assert sv._token_rows(cache[:, 7:8], 8, 1, 128)[1:] == (128 << 20, 128)
