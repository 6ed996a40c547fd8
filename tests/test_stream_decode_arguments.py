"""Arguments of the decoding example that are refused on the host (no GPU needed)."""

import types

import pytest


@pytest.mark.parametrize("prompts", [[[]], [[1, 2], [], [3]], []])
def test_empty_prompts_are_refused(prompts):
    from paper_2412_15803_amd import stream_decode as sd

    # Refused before the model is looked at any further.
    with pytest.raises(ValueError, match="prompt"):
        sd.generate(types.SimpleNamespace(device="cpu"), prompts, 1, 4, 32, 0)
