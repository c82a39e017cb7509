"""The optimizer's lists of tensors keep what they point to."""
import gc
import weakref

import pytest
import torch

from paper_2606_05484_amd import mapl

KINDS = dict(g=torch.float32, p=torch.float32, m=torch.uint8, v=torch.uint8, e=torch.uint8, p16=torch.bfloat16)


@pytest.mark.parametrize("name", KINDS)
@pytest.mark.parametrize("how", ["replaced", "cleared"])
def test_tensors_live_as_long_as_the_list_that_points_to_them(name, how):
    """Also where the caller's own list goes on to other tensors (gradients that are new every step)."""
    lists = {k: [torch.zeros(300, dtype=dt) for _ in range(3)] for k, dt in KINDS.items()}
    a = mapl.optim_params(**lists)
    first, at = weakref.ref(lists[name][0]), lists[name][0].data_ptr()
    if how == "replaced":
        lists[name][0] = torch.zeros(300, dtype=KINDS[name])
    else:
        lists[name].clear()
    gc.collect()
    assert first() is not None and first().data_ptr() == at == getattr(a.array[0], name)
    del a
    gc.collect()
    assert first() is None


def test_any_sequence_will_do():
    t = [torch.zeros(n) for n in (5, 300)]
    a = mapl.optim_params(tuple(t), p=torch.nn.ParameterList(t), weight_decay=(0.0, 0.5))
    assert [x.n for x in a.array] == [5, 300] and [x.weight_decay for x in a.array] == [0.0, 0.5]
