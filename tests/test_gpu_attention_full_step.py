"""Steps of the transformer blocks with attention over more than 256 keys a sequence (where the gradient's delta comes
from the stored output), and of one block at full size, against the oracle in every ordering."""
import pytest

from test_gpu_attention_training import _window
from workloads import get_config, reduced_config

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_sequences(gpu, progress, dtype):
    cfg = reduced_config("attn12", dtype=dtype)
    cfg["batch"] = 640
    cfg["attention"]["seq_len"] = 320
    _window(gpu, cfg, 1, progress)


@pytest.mark.timeout(300)
def test_full_size_block(gpu, progress):
    """4 x 1024 rows of width 1024, 16/4 heads of 64, one block deep."""
    cfg = dict(get_config("attn12"), blocks=1)
    progress("attn12, one block: oracle and three orderings")
    _window(gpu, cfg, 0, progress)
