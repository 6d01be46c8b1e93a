"""Rows into pages whose heads several CTAs share, where a thread does not hold its place of the page: more places than threads, pieces of less than 16 bytes."""
import pytest

from test_gpu_layer_ops import BF16, F32
from test_gpu_pages import test_append as check_append

pytestmark = pytest.mark.gpu

# (B, H, d, page, dtype, 8 bits, rotated channels (0: none), interleaved, tokens of each call, layout)
APPENDS = [
    (1, 9, 256, 128, BF16, True, 256, False, [300, 1, 5], "tokens"), (1, 10, 128, 128, F32, True, 128, False, [200, 3, 100], "heads"), (2, 9, 80, 64, BF16, True, 20, False, [70, 1, 60], "tokens"),
    (1, 13, 256, 128, F32, True, 0, False, [129, 128], "heads"), (1, 9, 72, 32, BF16, False, 10, False, [40, 2], "heads"), (1, 17, 256, 128, F32, False, 200, True, [260, 1], "tokens"),
    (3, 5, 48, 128, BF16, True, 36, False, [128, 127, 2], "heads"), (1, 21, 128, 128, F32, True, 128, True, [5, 250], "tokens"),
]


@pytest.mark.parametrize("b, h, d, p, dtype, eight, r, inter, calls, layout", APPENDS, ids=lambda x: str(x) if isinstance(x, (int, str)) else None)
def test_heads_shared_out(b, h, d, p, dtype, eight, r, inter, calls, layout):
    check_append(b, h, d, p, dtype, eight, r, inter, calls, layout)
