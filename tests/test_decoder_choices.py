"""What the decoder's choices refuse, before anything reaches a GPU."""
import pytest
import torch


def test_activations_have_a_name():
    from paper_2301_12017_amd import decoder as dec
    z = torch.zeros((8, 8), dtype=torch.float16)
    for name in ("16", None, "prompt"):
        with pytest.raises(ValueError):
            dec.DecoderLayer(*[z] * 12, heads=1, kv_heads=1, blocks=1, weights="mx4", activations=name)


@pytest.mark.parametrize("kw", [{"group": 64}, {"mode": 0}, {"mode": 1}, {"group": 0, "mode": 1}])
def test_microscaled_weights_have_no_mode_and_no_groups(kw):
    from paper_2301_12017_amd import decoder as dec
    with pytest.raises(ValueError, match="no mode"):
        dec.quantized(torch.zeros((8, 64), dtype=torch.float16), "mx4", **kw)
    z, books = torch.zeros((8, 64), dtype=torch.float16), dec.Books(3, 64, 12, 16, device="cpu")
    with pytest.raises(ValueError, match="no mode"):
        dec.DecoderLayer(torch.zeros((192, 8), dtype=torch.float16), z, z, z, z, z, z, z, z, z, z, z, heads=1, kv_heads=1, blocks=1, weights="mx4", **kw)
    if "group" in kw:
        with pytest.raises(ValueError, match="no mode"):
            dec.Decoder([], z, torch.zeros((64, 64), dtype=torch.float16), books, group=kw["group"], weights="mx4")
