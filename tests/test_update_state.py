"""What a step of the orthogonalised updates hands to the library, on the CPU: the call
itself is replaced by one that records its descriptors, and tensors of host memory take the
device's place."""
import numpy as np
import pytest
import torch

from paper_2501_08582_amd import train

ITEM = ("rows", "cols", "grad", "m", "master", "param", "rate", "decay")


@pytest.fixture
def calls(monkeypatch):
    seen = []

    def record(p, items, count, ws, dev):
        seen.append([{n: getattr(items[i], n) for n in ITEM} for i in range(count)])

    monkeypatch.setattr(train, "_dev", lambda *ts: torch.device("cpu"))
    monkeypatch.setattr(train, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(train, "_run_update", record)
    return seen


def made(shapes=((4, 30), (50, 3)), dtype=torch.bfloat16, own=False):
    masters = [torch.randn(s) for s in shapes]
    params = masters if own else [w.to(dtype) for w in masters]
    return train.OrthogonalUpdate(masters, params), [torch.randn(s) for s in shapes]


def addresses(seen, *names):
    return [tuple(item[n] for n in names) for item in seen[-1]]


def test_a_step_works_on_what_the_lists_hold(calls):
    """Restored momenta, other masters, another list."""
    opt, grads = made()
    opt.step(grads, 0.1)
    opt.momenta[1] = torch.ones(50, 3)
    opt.masters[0] = torch.zeros(4, 30)
    opt.params = [q.clone() for q in opt.params]
    opt.step(grads, 0.1)
    want = [(w.data_ptr(), m.data_ptr(), q.data_ptr(), g.data_ptr())
            for w, m, q, g in zip(opt.masters, opt.momenta, opt.params, grads)]
    assert addresses(calls, "master", "m", "param", "grad") == want
    assert addresses(calls, "rows", "cols") == [(4, 30), (50, 3)]


def test_a_step_follows_a_tensor_to_its_new_storage(calls):
    opt, grads = made()
    opt.step(grads, 0.1)
    opt.params[0].data = opt.params[0].data.clone()
    opt.momenta[0].set_(torch.ones(4, 30))
    opt.masters[1].data = torch.zeros(50, 3)
    opt.step(grads, 0.1)
    want = [(w.data_ptr(), m.data_ptr(), q.data_ptr()) for w, m, q in zip(opt.masters, opt.momenta, opt.params)]
    assert addresses(calls, "master", "m", "param") == want


def test_a_parameter_may_become_or_cease_to_be_its_own_master(calls):
    opt, grads = made(own=True)
    opt.step(grads, 0.1)
    assert addresses(calls, "param") == [(None,), (None,)]
    opt.params[0] = torch.zeros(4, 30)
    opt.step(grads, 0.1)
    assert addresses(calls, "param") == [(opt.params[0].data_ptr(),), (None,)]


@pytest.mark.parametrize("change,what", [
    (lambda o: o.momenta.__setitem__(0, torch.zeros(4, 31)), "momentum 0"),
    (lambda o: o.momenta.__setitem__(0, torch.zeros(4, 30, dtype=torch.float64)), "momentum 0"),
    (lambda o: o.masters.__setitem__(1, torch.zeros(3, 50)), "master 1"),
    (lambda o: o.params.__setitem__(0, torch.zeros(4, 30)), "param 0"),
    (lambda o: o.momenta.pop(), "momentum: expected 2"),
    (lambda o: o.momenta[0].untyped_storage().resize_(0), "released"),
])
def test_a_change_of_shape_type_or_count_is_refused(calls, change, what):
    opt, grads = made()
    opt.step(grads, 0.1)
    change(opt)
    for _ in range(2):
        with pytest.raises(ValueError, match=what):
            opt.step(grads, 0.1)
    assert len(calls) == 1


def test_memory_at_an_address_that_a_step_uses_is_not_handed_out_again(calls):
    """The storage of a replaced tensor stays until the next step has taken the new one's address: the
    same address is the same memory."""
    opt, grads = made()
    opt.step(grads, 0.1)
    was = opt.momenta[0].data_ptr()
    opt.momenta[0] = None
    opt.momenta[0] = torch.zeros(4, 30)
    assert opt.momenta[0].data_ptr() != was
    opt.step(grads, 0.1)
    assert calls[-1][0]["m"] == opt.momenta[0].data_ptr()


def rates(seen):
    return [(item["rate"], item["decay"]) for item in seen[-1]]


def test_the_weight_decay_may_change_at_one_lr(calls):
    opt, grads = made()
    opt.step(grads, 0.5)
    tall = (50 / 3) ** 0.5
    assert rates(calls) == [(0.5, 0.0), (0.5 * tall, 0.0)]
    opt.weight_decay = 0.25
    opt.step(grads, 0.5)
    assert rates(calls) == [(0.5, 0.125), (0.5 * tall, 0.125)]


@pytest.mark.parametrize("lr", [torch.tensor(0.5), np.array(0.5)])
def test_a_learning_rate_changed_in_place(calls, lr):
    opt, grads = made()
    opt.weight_decay = 1.0
    opt.step(grads, lr)
    lr *= 0.5
    opt.step(grads, lr)
    assert rates(calls)[0] == (0.25, 0.25)
    opt.step(grads, 0.25)
    assert rates(calls)[0] == (0.25, 0.25)


def test_a_step_counts_as_a_change_in_place(calls):
    """A graph that saved a parameter before the step refuses its backward after it, as after any change
    in place; detached views share the count."""
    opt, grads = made(((4, 30), (30, 5)), torch.float32)
    leaf = opt.params[0].detach().requires_grad_(True)
    opt.params[0] = leaf.detach()
    y = (leaf * leaf).sum()
    held = [*opt.masters, *opt.momenta, *opt.params]
    before = [t._version for t in held]
    opt.step(grads, 0.1)
    assert all(t._version > v for t, v in zip(held, before))
    with pytest.raises(RuntimeError, match="inplace operation"):
        y.backward()
    with torch.inference_mode():
        made(own=True)[0].step(grads[:1] + [torch.randn(50, 3)], 0.1)  # (such tensors have no count)
