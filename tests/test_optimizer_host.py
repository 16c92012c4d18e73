"""What AdamW hands to foremoe_adamw_step after its tensors or hyperparameters
changed, on the host: the library is replaced by a recorder, and CPU tensors
stand for device tensors."""
import gc
import weakref

import numpy as np
import pytest
import torch

from paper_2606_11867_amd import optimizer

F32, BF16 = torch.float32, torch.bfloat16


class Recorder:
    def __init__(self):
        self.calls = []

    def foremoe_adamw_step(self, records, n, pdt, gdt, bits, lr, b1, b2, eps, step, scale, zero, stream):
        self.calls.append(dict(pdt=pdt, gdt=gdt, lr=lr, step=step,
                               records=[{k: getattr(records[i], k) for k, _ in records[i]._fields_} for i in range(n)]))
        return 0


@pytest.fixture
def lib(monkeypatch):
    rec = Recorder()

    def vec(t, n, dtype, name, device):
        if t is None:
            return None
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}")
        if t.numel() != n:
            raise ValueError(f"{name}: {t.numel()} elements, {n} expected")
        return t.data_ptr()

    monkeypatch.setattr(optimizer._lib, "load", lambda: rec)
    monkeypatch.setattr(optimizer, "_vec", vec)
    monkeypatch.setattr(optimizer, "_stream", lambda device: 0)
    return rec


def _made(dtype=F32, grad=F32, n=(300, 70), **kw):
    ps, gs = [torch.zeros(k, dtype=dtype) for k in n], [torch.ones(k, dtype=grad) for k in n]
    return ps, gs, optimizer.AdamW(ps, gs, **kw)


@pytest.mark.parametrize("which", ["params", "grads"])
@pytest.mark.parametrize("old,new", [(F32, BF16), (BF16, F32)])
def test_new_memory_of_another_type_is_refused(lib, which, old, new):
    """The call's types are those of the start: it would read and write 4
    bytes an element of a tensor that now has 2."""
    ps, gs, opt = _made(**{"dtype" if which == "params" else "grad": old}, masters=False)
    opt.step()
    for t in ps if which == "params" else gs:
        t.data = t.data.to(new)
    for _ in range(2):
        with pytest.raises(TypeError):
            opt.step()
    assert len(lib.calls) == 1 and opt.n_steps == 1
    for t in ps if which == "params" else gs:  # and back
        t.data = t.data.to(old)
    opt.step()
    assert [r["param"] for r in lib.calls[-1]["records"]] == [p.data_ptr() for p in ps]
    assert [r["grad"] for r in lib.calls[-1]["records"]] == [g.data_ptr() for g in gs]


def test_a_refused_step_leaves_the_records_whole(lib):
    """The first gradient moved, the second became wrong; both go back to
    where they were: the next call uses that memory, not the one between."""
    ps, gs, opt = _made()
    opt.step()
    kept = [g.data for g in gs]
    gs[0].data = torch.zeros(300)
    gs[1].data = torch.zeros(71)
    with pytest.raises(ValueError):
        opt.step()
    for g, k in zip(gs, kept):
        g.data = k
    opt.step()
    assert [r["grad"] for r in lib.calls[-1]["records"]] == [g.data_ptr() for g in gs]


def test_moved_tensors_keep_their_old_memory_until_the_next_step(lib):
    """A freed block could come back at the same address as something
    smaller, which addresses would not show."""
    array = np.ones(300, dtype=np.float32)
    ps, gs = [torch.zeros(300)], [torch.from_numpy(array)]
    opt = optimizer.AdamW(ps, gs)
    alive = weakref.ref(array)
    del array
    gs[0].data = torch.full((300,), 2.0)
    gc.collect()
    assert alive() is not None
    opt.step()
    gc.collect()
    assert alive() is None and lib.calls[-1]["records"][0]["grad"] == gs[0].data_ptr()


def test_weight_decay_counts_from_the_next_step(lib):
    ps, gs, opt = _made(weight_decay=0.1)
    opt.step()
    opt.weight_decay[1] = 0.3
    opt.step()
    opt.weight_decay = [0.0, 0.5]
    opt.lr = 0.7
    opt.step()
    got = [[r["weight_decay"] for r in c["records"]] for c in lib.calls]
    assert got == [[0.1, 0.1], [0.1, 0.3], [0.0, 0.5]]
    assert [c["lr"] for c in lib.calls] == [1e-3, 1e-3, 0.7]
    opt.weight_decay = 0.25  # one for all
    opt.step()
    assert [r["weight_decay"] for r in lib.calls[-1]["records"]] == [0.25, 0.25]
    with pytest.raises(ValueError):
        opt.weight_decay = [1.0]


@pytest.mark.parametrize("name", ["params", "grads", "masters", "states"])
def test_tensors_are_exchanged_by_new_memory_only(lib, name):
    """A tensor put in another's place would not be seen, and the old one's
    memory, which the records hold, could be freed."""
    ps, gs, opt = _made(dtype=BF16)
    held = getattr(opt, name)
    with pytest.raises(TypeError):
        held[0] = held[1]
    with pytest.raises(AttributeError):
        setattr(opt, name, held)
    with pytest.raises(AttributeError):  # records of the other width are read differently
        opt.state_bits = 8


@pytest.mark.gpu
def test_new_memory_of_another_type_is_refused_on_the_device(gpu):
    p, g = torch.zeros(300, device=gpu), torch.ones(300, device=gpu)
    opt = optimizer.AdamW([p], [g], lr=0.1)
    opt.step()
    p.data = p.data.to(BF16)
    beside = torch.full((600,), 3.0, device=gpu)
    with pytest.raises(TypeError):
        opt.step()
    p.data = p.data.float()
    g.data = g.data.to(BF16)
    with pytest.raises(TypeError):
        opt.step()
    g.data = g.data.float()
    opt.step()
    assert opt.n_steps == 2 and torch.all(p < -0.19) and torch.all(beside == 3.0)
