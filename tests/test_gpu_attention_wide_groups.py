"""Decoding with as many query heads to a key head, and as many buckets, as the call takes."""
import pytest

from test_gpu_attention import test_against_definition as against_definition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [(1, 1, 700, 32, 1, 128, True, 256, 1024, "append"), (1, 1, 600, 33, 1, 96, False, 256, 129, None),
                               (2, 1, 520, 40, 1, 128, True, 200, 1024, "append"), (1, 1, 600, 28, 1, 128, False, 256, 1000, None)], ids=str)
def test_many_heads_and_buckets(c, dtype):
    against_definition(c, dtype)
