"""Which tile of which environment and heads a workgroup of attention takes, where environments and heads are few enough that an XCD's workgroups go
through all of its heads tile by tile (a multiple of eight of them, up to 128), and next to that: against the definition in 64 bits."""
import pytest
from test_gpu_attn import _torch, define, make, near, run

pytestmark = pytest.mark.gpu

# T, S, N, H, KV, D, B, window, p_first: forward and queries go by environments x heads / (heads that share a tile), keys by environments x heads of keys
SHAPES = [
    (200, 260, 4, 4, 2, 32, 8, 260, 0.01),     # 8 and 8, seven and five tiles
    (130, 130, 8, 2, 2, 16, 0, 130, 0.0),      # 16 and 16, three tiles
    (150, 170, 8, 8, 1, 40, 6, 100, 0.02),     # 16 and 8, ten and three tiles
    (200, 200, 8, 2, 1, 128, 5, 200, 0.005),   # 8 and 8, the forward by 128 rows
    (70, 70, 8, 16, 16, 8, 4, 70, 0.0),        # 128 and 128
    (70, 70, 17, 8, 8, 8, 4, 70, 0.0),         # 136 and 136: too many
    (140, 140, 3, 4, 4, 16, 4, 140, 0.01),     # 12 and 12: no multiple
    (1100, 1100, 8, 1, 1, 16, 3, 1100, 0.002),   # 8 and 8, cut into chunks
    (600, 1200, 8, 4, 2, 64, 12, 1200, 0.0),     # 16 and 16, cut, two heads to a tile
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(v) for v in s))
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_every_tile_is_there(kind, shape):
    c = make(getattr(_torch(), kind), *shape)
    want, bound = define(c)
    got = run(c)
    for k in got:
        near(got[k], want[k], bound[k], k)
