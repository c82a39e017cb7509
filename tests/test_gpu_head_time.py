"""What head_step's printed time covers, whatever the optimizer: the gradients and the update."""
import pytest
import torch

from paper_2606_05484_amd import head_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("optimizer", ["sgd", "adamw", "adamw8"])
def test_the_update_is_timed(optimizer, monkeypatch, capsys):
    """Between a step's two events the gradients are made, the head moves, and so does its bf16 copy."""
    seen, heads = [], []

    class Event(torch.cuda.Event):
        def record(self, *args):
            seen.append("record")
            if heads:
                head, copy = heads[-1]
                seen.append((head.clone(), copy.clone()))
            return super().record(*args)

    Step = head_step.HeadStep
    run = Step.gradients

    def gradients(self, *args, **kw):
        seen.append("gradients")
        return run(self, *args, **kw)

    for name in ("SGD", "AdamW"):
        kind = getattr(head_step, name)
        start = kind.__init__

        def init(self, params, grads, copies=(), *args, _start=start, **kw):
            heads.append((params["W"], dict(copies)["W"]))
            return _start(self, params, grads, copies, *args, **kw)

        monkeypatch.setattr(kind, "__init__", init)
    monkeypatch.setattr(Step, "gradients", gradients)
    monkeypatch.setattr(head_step.torch.cuda, "Event", Event)
    head_step.main(["--tokens", "200", "--d", "64", "--r", "64", "--vocabulary", "501", "--micro", "1", "--steps", "2", "--optimizer", optimizer])
    assert [x for x in seen if isinstance(x, str)] == ["record", "gradients", "record"] * 2
    values = [x for x in seen if not isinstance(x, str)]
    for (before, copy_before), (after, copy_after) in zip(values[::2], values[1::2]):
        assert not torch.equal(before, after) and torch.equal(copy_after, after.to(torch.bfloat16))
        assert torch.equal(copy_before, before.to(torch.bfloat16))


def test_plain_steps():
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    params, grads = ({"W": rn(50, 64), "w": rn(64)} for _ in range(2))
    W = torch.zeros(50, 64, dtype=torch.bfloat16, device="cuda")
    before = {k: v.clone() for k, v in params.items()}
    head_step.SGD(params, grads, {"W": W}, 0.5).step()
    for k, v in params.items():
        assert ((v.double() - (before[k].double() - 0.5 * grads[k].double())).abs() <= 2.0 ** -24 * v.double().abs() * 1.01).all()
    assert torch.equal(W, params["W"].to(torch.bfloat16))
