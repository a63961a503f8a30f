"""Which kinds of layers the probe has (no GPU needed)."""
import pytest

from paper_2608_19659_amd import probe


def test_kinds_of_attention(capsys):
    for kind in probe.ATTENTIONS:
        probe.Decoder(attention=kind).check(8)
    with pytest.raises(ValueError, match="attention"):
        probe.Decoder(attention="none").check(1)
    with pytest.raises(SystemExit) as e:
        probe.main(["--attention", "none"])
    assert e.value.code == 2
