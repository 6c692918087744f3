"""What a model's window may be, on the host: refused before a device is touched."""
import pytest

from paper_2401_10652_amd import inputs as I


@pytest.mark.parametrize("kw", [dict(window=-1), dict(window=(1 << 30) + 1), dict(window=8, sinks=-1), dict(window=8, sinks=(1 << 30) + 1), dict(sinks=-1)])
def test_refusals(kw):
    from paper_2401_10652_amd.decode import Decoder
    cfg = I.TransformerConfig("decoder_1l", 11, 1, 8, 64, 2, 128, True, "f32", None, batch=1)
    _, layers = I.transformer_inputs(cfg)
    with pytest.raises(ValueError, match="window"):
        Decoder(cfg, layers, 2, 100, **kw)
