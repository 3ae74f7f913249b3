"""What the decoder's choices refuse, before anything reaches a GPU."""
import pytest
import torch


def test_activations_have_a_name():
    from paper_2301_12017_amd import decoder as dec
    z = torch.zeros((8, 8), dtype=torch.float16)
    for name in ("16", None, "prompt"):
        with pytest.raises(ValueError):
            dec.DecoderLayer(*[z] * 12, heads=1, kv_heads=1, blocks=1, weights="mx4", activations=name)
