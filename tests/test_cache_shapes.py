"""The binding of the operators over an uncompressed cache looks at shapes, not only at numbers of elements (no GPU needed: the device
comes last among the checks)."""
import pytest
import torch


@pytest.fixture(scope="module")
def xkv():
    from paper_2503_18893_b200 import build
    build.build()
    from paper_2503_18893_b200 import xkv as m
    return m


G, BATCH, H_KV, H_Q, D, CAP, N = 2, 3, 4, 8, 64, 100, 5
ORDER, DEVICE = "K: .*axes in another order", "K: .*current CUDA device"


def config(xkv, **over):
    return xkv.make_cache_config(**dict(dict(G=G, batch=BATCH, H_kv=H_KV, H_q=H_Q, d_h=D, cap=CAP), **over))


@pytest.mark.parametrize("shape,what", [
    ((G, BATCH, H_KV, CAP, D), DEVICE), ((G * BATCH, H_KV, CAP, D), DEVICE), ((G * BATCH * H_KV, CAP, D), DEVICE), ((G * BATCH * H_KV * CAP * D,), DEVICE),
    ((1, G, BATCH, 1, H_KV, CAP, D), DEVICE), ((G, BATCH, 2, 2, CAP, 2, D // 2), DEVICE), ((G * BATCH, 2, 2, CAP, D), DEVICE),
    ((G, BATCH, CAP, H_KV, D), ORDER), ((BATCH, G, H_KV, CAP, D), ORDER), ((G, BATCH, H_KV, D, CAP), ORDER), ((CAP, G * BATCH * H_KV, D), ORDER),
    ((G, CAP, BATCH, H_KV, D), ORDER)])
def test_a_cache(xkv, shape, what):
    K = torch.zeros(shape, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match=what):
        xkv.xkv_tree_commit(config(xkv), 0, G, K, K, None, None, None, N)
    with pytest.raises(ValueError, match=what):
        xkv.xkv_evict_compact(config(xkv), 0, G, K, K, None, 7)


def test_a_single_layer_and_sequence(xkv):
    cfg = config(xkv, G=1, batch=1)
    for shape, what in (((H_KV, CAP, D), DEVICE), ((1, 1, H_KV, CAP, D), DEVICE), ((1, CAP, H_KV, D), ORDER), ((1, 1, CAP, H_KV, D), ORDER)):
        K = torch.zeros(shape, dtype=torch.bfloat16)
        with pytest.raises(ValueError, match=what):
            xkv.xkv_tree_commit(cfg, 0, 1, K, K, None, None, None, N)


@pytest.mark.parametrize("shape,what", [((G, BATCH, N, H_Q, D), "current CUDA device"), ((G * BATCH, N, H_KV, H_Q // H_KV, D), "current CUDA device"),
                                        ((G, BATCH, H_Q, N, D), "another order"), ((G, N, BATCH, H_Q, D), "another order"),
                                        ((G, BATCH, N, H_Q + 1, D), "another number of elements")])
def test_queries(xkv, shape, what):
    q = torch.zeros(shape, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q: .*" + what):
        xkv.xkv_tree_attend(config(xkv), 0, G, q, N, None, None, None, None, None, None, None)


def test_weights_and_positions(xkv):
    for shape, what in (((G, BATCH, H_KV, CAP), "current CUDA device"), ((G, BATCH, CAP, H_KV), "another order"), ((BATCH, G, H_KV, CAP), "another order")):
        with pytest.raises(ValueError, match="weights: .*" + what):
            xkv.xkv_evict_select(config(xkv), 0, G, torch.zeros(shape), None, None, None, 7, None)


def test_sizes_that_are_none(xkv):
    """Sizes of zero or below are refused, whatever the tensors are."""
    for over in (dict(G=0), dict(batch=-1), dict(cap=0), dict(G=-1, batch=-1)):
        K = torch.zeros((H_KV, CAP, D), dtype=torch.bfloat16)
        with pytest.raises((ValueError, xkv.XKVError)):
            xkv.xkv_tree_commit(config(xkv, **over), 0, 1, K, K, None, None, None, N)
