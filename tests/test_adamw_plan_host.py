"""What AdamW's plan takes and refuses on the host (no GPU needed)."""
import pytest

from paper_2401_06197_amd import binding as dcn


def plan(count=3):
    records = (dcn.AdamwTensor * count)()
    p = dcn.AdamwPlan(records, (), None, 32, dcn.DCNV4_F32)
    p.set(lr=[0.1, 0.2, 0.3], weight_decay=0.5)
    return p


def rates(p):
    return [(r.lr, r.weight_decay) for r in p.records]


def test_set_takes_a_number_or_one_for_each():
    p = plan()
    assert rates(p) == [(0.1, 0.5), (0.2, 0.5), (0.3, 0.5)]
    p.set(weight_decay=(0, 1, 2))
    p.set(lr=7)
    assert rates(p) == [(7.0, 0.0), (7.0, 1.0), (7.0, 2.0)]


@pytest.mark.parametrize("kw", [{"lr": 1.0, "weight_decay": [1.0, 2.0]}, {"lr": [1.0, 2.0, 3.0], "weight_decay": "much"}, {"lr": 1.0, "weight_decay": [0.0, 1.0, object()]},
                                {"lr": [1.0], "weight_decay": 2.0}])
def test_a_refused_set_changes_nothing(kw):
    p = plan()
    before = rates(p)
    with pytest.raises((ValueError, TypeError)):
        p.set(**kw)
    assert rates(p) == before
