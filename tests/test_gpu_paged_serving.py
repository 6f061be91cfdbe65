"""PagedCache and DecoderLayer.step(): caches that are another layer's."""
import pytest
import torch

from paper_2411_09909_amd import binding, layer, synth
from tests import gpu_util as G
from tests.test_gpu_paged import FORMATS
from tests.test_gpu_paged_layer import make_layer, ones

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,head_dim", [(8, 1, 64), (8, 4, 64), (4, 1, 128), (4, 2, 128)])
def test_step_refuses_a_cache_of_other_heads(heads, kv_heads, head_dim):
    """Fewer or smaller heads would read keys and values out of the wrong columns of the projection."""
    cfg = layer.LayerConfig(d_model=512, n_heads=8, n_kv_heads=2, head_dim=64, d_ff=1024)
    _, lay = make_layer(cfg, *FORMATS["amxfp4_e5m2"])
    other = layer.LayerConfig(d_model=512, n_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim, d_ff=1024)
    cache = layer.PagedCache(other, lay.fmt, 2, 8, 128, 16)
    before = [t.clone() for t in cache.pools[0]]
    with pytest.raises(binding.AmxError, match="the layer has 2 of 64"):
        lay.step(G.to_dev_bf16(synth.layer_input(2, cfg.d_model, seed=1)), cache, cache.plan(ones(1, 1), 2))
    assert all(torch.equal(a, b) for a, b in zip(before, cache.pools[0]))
