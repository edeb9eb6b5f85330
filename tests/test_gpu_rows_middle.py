"""The experts' middle tiles: the checks of a hundred rows an expert at seventy."""
import pytest

import test_gpu_rows_tiles as tiles

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,hidden,inter", [("bf16", 1024, 130), ("bf16", 512, 400), ("int8", 1024, 136)])
def test_many_experts_with_seventy_rows(lib, monkeypatch, fmt, hidden, inter):
    monkeypatch.setattr(tiles, "MIDDLE", [70, 97, 0, 128, 65, 33, 129, 64, 1, 90] * 9)
    tiles.test_many_experts_with_a_hundred_rows(lib, fmt, hidden, inter)
