"""Head counts and widths at the ends of what a model may have, for trees, weights,
kept tokens and evictions."""
import pytest
import torch

import prompt_ref
import test_gpu_keep as keep
import test_gpu_tree as tree
import test_gpu_weights as weights
from paper_2606_24506_amd import crosspool as cpl
from token_ref import make_tree

pytestmark = pytest.mark.gpu

WIDE = {
    "gqa256x256d64": dict(kind=cpl.CP_KIND_GQA, n_q_heads=256, n_kv_heads=256, head_dim=64),
    "gqa256x2d128": dict(kind=cpl.CP_KIND_GQA, n_q_heads=256, n_kv_heads=2, head_dim=128),
    "gqa51x17d128": dict(kind=cpl.CP_KIND_GQA, n_q_heads=51, n_kv_heads=17, head_dim=128),
    "gqa3x3d512": dict(kind=cpl.CP_KIND_GQA, n_q_heads=3, n_kv_heads=3, head_dim=512),
    "mla256": dict(kind=cpl.CP_KIND_MLA, n_q_heads=256, n_kv_heads=1, latent_dim=512, rope_dim=64, softmax_scale=0.07),
    "mla1": dict(kind=cpl.CP_KIND_MLA, n_q_heads=1, n_kv_heads=1, latent_dim=512, rope_dim=64, softmax_scale=0.07),
    "mla9l512r512": dict(kind=cpl.CP_KIND_MLA, n_q_heads=9, n_kv_heads=1, latent_dim=512, rope_dim=512, softmax_scale=0.03),
}


@pytest.mark.parametrize("name", sorted(WIDE))
def test_head_counts(name, monkeypatch):
    print(f"[case] heads {name}", flush=True)
    monkeypatch.setitem(prompt_ref.GEOMS, name, WIDE[name])
    sc = prompt_ref.Scene(name, [40, 75], page_tokens=4, seed=3, room=20)
    tree.verify(sc, [make_tree(1, 1), make_tree(9, 2)], name)
    weights.verify(sc, [1, 9], name, decay=0.5, pad=3)
    weights.verify(sc, [17, 40], name, num_splits=2)
    keep.evict(sc, sc.ids, [r[None] for r in sc.rows], [20, 33], "steps", 3, 5)
    sc.close()
    sc = prompt_ref.Scene(name, [40], page_tokens=4, seed=4)
    sc.pool.keep(sc.ids, [6], [4], [1, 9, 20, 33])
    assert torch.equal(sc.held(sc.ids[0], 10), torch.cat([sc.rows[0][:6], sc.rows[0][6:][[1, 9, 20, 33]]]))
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16", "mla4l64r0"])
def test_pages_past_4_gib(name):
    print(f"[case] far pages {name}", flush=True)
    sc = prompt_ref.Scene(name, [700, 900], seed=5, room=20, pool_bytes=12 << 30)
    far = [int((sc.pool.pages(i).astype("int64") << 8).max()) for i in sc.ids]
    assert max(far) > 1 << 32
    tree.verify(sc, [make_tree(5, 1), make_tree(40, 2)], name)
    weights.verify(sc, [1, 40], name)
    weights.verify(sc, [130, 3], name, num_splits=2)
    b = sc.pool.open(sc.model, 920)
    sc.pool.fork([sc.ids[1]], [b])
    keep.evict(sc, [b], [sc.rows[1][None]], [300], "normal", 3, 5)
    keep.evict(sc, sc.ids, [r[None] for r in sc.rows], [200, 333], "normal", 3, 5)
    sc.ids.append(b)
    sc.close()
