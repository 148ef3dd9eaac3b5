"""4-bit networks and networks with a teacher, on the host: codes handed over,
what is refused, and what a step calls (no GPU needed)."""

import pytest
import torch

from paper_2607_14672_gb300 import build, configs, dstd, net


@pytest.fixture(scope="module", autouse=True)
def lib():
    try:
        build.build()
    except RuntimeError:
        pytest.skip("the library does not build here")


def network(sizes=(20, 40, 10), mode="mx4", batch=2):
    cfg = configs.config2(batch=batch, M=8)
    layer = cfg["layers"][0]
    cfg["layers"] = [dict(layer, W=torch.zeros(b, a).numpy()) for a, b in zip(sizes, sizes[1:])]
    return net.DenseNet(cfg, mode, device="cpu")


def with_codes(n):
    for i, x in enumerate(n.Wq + n.w_scale):
        x.fill_(i + 1)
    n.has_codes = True
    return n


def test_codes_are_taken_over():
    a, b = with_codes(network()), network(batch=5)
    assert [tuple(q.shape) for q in a.Wq] == [(40, 16), (10, 32)] and [s.numel() for s in a.w_scale] == [512, 512]
    b.take_codes(a)
    assert b.has_codes
    assert all(torch.equal(x, y) for x, y in zip(a.Wq + a.w_scale, b.Wq + b.w_scale))


def test_codes_of_another_kind_are_refused():
    a = network()
    for other in (with_codes(network(mode="q8")), network(), network(mode="x3"), with_codes(network((20, 41, 10)))):
        with pytest.raises(ValueError):
            a.take_codes(other)
    with pytest.raises(ValueError):
        network(mode="q8").take_codes(with_codes(network()))
    with pytest.raises(RuntimeError):
        a.serve()
    assert not a.has_codes


def test_teacher_is_refused_where_there_are_no_logits():
    n = network(mode="x3")
    with pytest.raises(RuntimeError):
        n.set_teacher(torch.zeros(2, 3), torch.zeros(2, 3))
    n.cfg["tau_soft"] = None
    with pytest.raises(ValueError):
        n.learn_from(3)
    with pytest.raises(ValueError):
        n.answers(torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32))
    assert n.record is None
    n = network(mode="x3")
    for K in (0, 257):
        with pytest.raises(ValueError):
            n.learn_from(K)
    n.learn_from(3)
    for top, index in ((torch.zeros(2, 2), torch.zeros(2, 3)), (torch.zeros(2, 3), torch.zeros(3)), (torch.zeros(3), torch.zeros(2, 3))):
        with pytest.raises(ValueError):
            n.set_teacher(top, index)


@pytest.mark.parametrize("mode", ["mx4", "x3"])
@pytest.mark.parametrize("labels", [True, False])
def test_what_a_step_calls(monkeypatch, mode, labels):
    calls = []
    for name in ("dense_fwd", "dense_fwd_mx4", "dense_fwd_ce", "ce_loss", "dense_bwd", "quantize_mx4", "distill_loss"):
        monkeypatch.setattr(dstd, name, lambda *a, _n=name, **k: calls.append((_n, k.get("accumulate"))))
    n = network(mode=mode)
    n.learn_from(3, weight=2.0, labels=labels)
    n.set_teacher([[1.0, 0.5, 0.0]] * 2, [[1, 2, -1]] * 2)
    assert n.record[0].tolist() == [[1.0, 0.5, 0.0]] * 2 and n.record[1].tolist() == [[1, 2, -1]] * 2
    n.step()
    names = [c[0] for c in calls]
    assert names.count("distill_loss") == 1 and ("distill_loss", labels) in calls
    assert names.count("ce_loss") + names.count("dense_fwd_ce") == (1 if labels else 0)
    first = min(i for i, x in enumerate(names) if x == "dense_bwd")
    assert names.index("distill_loss") < first
    if labels:
        assert max(i for i, x in enumerate(names) if x in ("ce_loss", "dense_fwd_ce")) < names.index("distill_loss")


def test_a_record_is_taken_whole_or_not_at_all():
    n = network(mode="x3")
    n.learn_from(3)
    logits, classes = torch.ones(2, 3), torch.ones(2, 3, dtype=torch.int32)
    n.set_teacher(logits, classes)
    for bad in ((logits + 1, classes[:, :2]), (logits[:1] + 1, classes)):
        with pytest.raises(ValueError):
            n.set_teacher(*bad)
        assert torch.equal(n.record[0], logits) and torch.equal(n.record[1], classes)
