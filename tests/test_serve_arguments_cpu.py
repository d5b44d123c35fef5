"""What a decoder refuses when it is made (no GPU: nothing is launched)."""

import pytest

from paper_2506_03781_gb300 import serve, synth
from tests.test_serve_cpu import pool


@pytest.mark.parametrize("more", [dict(window=-1), dict(sinks=-1), dict(window=4, sinks=-2)])
def test_windows_and_sinks_are_checked_before_a_page_is_taken(more):
    shape = synth.BLOCKS["tiny"]
    with pytest.raises(ValueError, match="window"):
        serve.BlockDecoder(shape, {}, 64, pool(), **more)
