"""examples/decode_layer.py: the projections, the cache and its eviction together, and its last attention against the cache as it reads back."""
import os
import runpy

import pytest

pytestmark = pytest.mark.gpu

EXAMPLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_layer.py")


def test_decode_layer():
    import torch
    import paper_2511_04477_amd as spqt
    assert torch.cuda.is_available()
    assert spqt.lib()
    main = runpy.run_path(EXAMPLE)["main"]
    layer = main("--hidden 512 --q-heads 8 --kv-heads 2 --head-dim 64 --prompt 90 --steps 120 --budget 70 --recent 16".split())
    # 210 tokens against a budget of 70: cut down at 134, every time
    assert layer.position == 210 and layer.evictions == 2 and layer.in_cache == int(layer.lengths) == 82
    kept = layer.kept.cpu()
    assert bool((kept[..., 1:] > kept[..., :-1]).all()) and bool((kept[..., -16:] == torch.arange(118, 134)).all())
    # what the last step saw is what is in the cache: read back in fp16, each value within half of fp16's step of itself of what attention used
    k, v = (t.double().cpu() for t in layer.cached())
    q, out = (t[0, 0].double().cpu() for t in layer.last)
    for j in range(8):
        h = j // 4
        p = torch.softmax(k[:, h] @ q[j] * 64 ** -0.5, dim=0)
        want = p @ v[:, h]
        # scores: 2^-11 of sum |q| |k| / 8; probabilities twice that; values and the output 2^-11 of themselves
        off = 2 * 2.0 ** -11 * float((k[:, h].abs() @ q[j].abs()).max()) * 64 ** -0.5
        bound = (p @ v[:, h].abs()) * (off + 2.0 ** -11) + 2.0 ** -11 * want.abs() + 2.0 ** -14
        assert bool(((out[j] - want).abs() <= bound).all())
    # every query head has given away one unit of weight per step since its kv head's tokens came; what was dropped took its share along
    total = layer.seen[layer.table[0].long()].sum(dim=(0, 2))
    assert bool(torch.isfinite(total).all()) and bool((total > 0).all()) and bool((total <= 4 * 210).all())
