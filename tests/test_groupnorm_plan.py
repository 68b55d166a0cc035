"""The group norm's division of an image into chunks, by the workspace that it asks for; without a device the plan is that of one compute unit."""
import pytest

import paper_2411_00288_amd as ss


@pytest.mark.parametrize("images,pixels,channels", [(1, 1 << 22, 2048), (1, 1 << 20, 16384), (3, 1 << 18, 1032), (1, 1 << 24, 64), (2000, 1 << 20, 256)])
def test_a_thread_adds_at_most_512_rows(images, pixels, channels):
    ws = ss.ss_groupnorm_workspace_bytes(ss.make_groupnorm_desc(channels, 1, ss.SS_F32), images, pixels)
    chunks, slots = ws // (images * channels * 8), 256 // min((channels + 7) // 8, 256)
    assert pixels / chunks / slots <= 513
