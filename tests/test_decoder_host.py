"""What the decoder refuses before anything reaches a GPU."""
import pytest
import torch


@pytest.mark.parametrize("context, block, room", [(500, 16, 512), (512, 16, 512), (1, 128, 128), (129, 128, 256)])
def test_positions_for_every_token_that_blocks_can_hold(context, block, room):
    """The bookkeeping serves tokens up to whole blocks: each of their positions needs its embedding."""
    from paper_2301_12017_amd import decoder as dec
    books = dec.Books(3, context, 12, block, device="cpu")
    assert books.table.shape[1] * block == room and books.context == room
    tokens = torch.zeros((8, 64), dtype=torch.float16)
    with pytest.raises(ValueError):
        dec.Decoder([], tokens, torch.zeros((room - 1, 64), dtype=torch.float16), books)
