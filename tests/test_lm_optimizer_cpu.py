"""What an AdamW step hands to the library, without a GPU: the launch is replaced by one that keeps the records, everything else is
the optimiser's own.  Every address has to be that of the tensors as they are at the time of the step."""
import ctypes as C
import gc
import weakref

import pytest
import torch

import paper_2505_05086_amd as asi
from paper_2505_05086_amd import binding as B, lm

SIZES = [(300, 3), (256,), (7,)]


class _Launches:
    """In place of the library: what it was called with."""

    def __init__(self):
        self.records = []

    def asi_adamw(self, count, records, bits, *rest):
        size = C.sizeof(B.AdamwTensor) * count
        data = records[:size] if isinstance(records, bytes) else C.string_at(records, size)
        self.records = list((B.AdamwTensor * count).from_buffer_copy(data))
        self.bits = bits
        return 0


@pytest.fixture
def launches(monkeypatch):
    fake = _Launches()
    monkeypatch.setattr(B, "lib", lambda: fake)
    monkeypatch.setattr(lm, "_place", lambda *tensors: -1)
    monkeypatch.setattr(lm, "_stream", lambda device: 0)
    return fake


def _made(bits=32, master=False, dtype=torch.float32):
    g = torch.Generator().manual_seed(1)
    params = [torch.nn.Parameter(torch.randn(s, generator=g).to(dtype)) for s in SIZES]
    opt = asi.AdamW(params, lr=1e-2, weight_decay=0.1, state_bits=bits, master=master)
    _gradients(params)
    return params, opt


def _gradients(params):
    for p in params:
        p.grad = torch.ones_like(p)


def _agree(fake, opt, params):
    """The records of the last step are those of the tensors as they are."""
    bits = opt.param_groups[0]["state_bits"]
    assert fake.bits == bits and len(fake.records) == len(params)
    at = lambda t: None if t is None else t.data_ptr() or None  # noqa: E731
    for r, p in zip(fake.records, params):
        s = opt.state[p]
        assert (r.param, r.grad, r.count) == (at(p), at(p.grad), p.numel())
        assert (r.param_dtype, r.grad_dtype) == tuple(B.ASI_F32 if t.dtype == torch.float32 else B.ASI_BF16 for t in (p, p.grad))
        assert (r.lr, r.weight_decay) == (opt.param_groups[0]["lr"], opt.param_groups[0]["weight_decay"])
        assert r.master == at(s.get("master"))
        assert r.exp_avg == at(s["exp_avg"]) and r.exp_avg_sq == at(s["exp_avg_sq" if bits == 32 else "exp_avg_sqrt"])
        assert r.exp_avg_scale == at(s.get("exp_avg_scale")) and r.exp_avg_sq_scale == at(s.get("exp_avg_sqrt_scale"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_records_are_those_of_the_tensors(launches, bits, dtype):
    params, opt = _made(bits, True, dtype)
    for step in range(3):
        opt.param_groups[0]["lr"] = 0.1 * (step + 1)
        opt.step()
        _agree(launches, opt, params)
        assert ("master" in opt.state[params[0]]) == (dtype == torch.bfloat16)
        _gradients(params)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_removed_master_is_made_anew(launches, bits):
    params, opt = _made(bits, True, torch.bfloat16)
    opt.step()
    with torch.no_grad():
        params[0].fill_(0.5)
    old = weakref.ref(opt.state[params[0]]["master"])
    del opt.state[params[0]]["master"]
    gc.collect()
    assert old() is None
    opt.step()
    _agree(launches, opt, params)
    assert (opt.state[params[0]]["master"] == 0.5).all()


@pytest.mark.parametrize("bits,name", [(32, "exp_avg"), (32, "exp_avg_sq"), (8, "exp_avg"), (8, "exp_avg_sqrt"), (8, "exp_avg_scale"), (8, "exp_avg_sqrt_scale"),
                                       (32, "master"), (8, "master")])
def test_a_replaced_state_is_used(launches, bits, name):
    params, opt = _made(bits, name == "master", torch.bfloat16)
    opt.step()
    old = opt.state[params[1]][name]
    opt.state[params[1]][name] = old.clone()
    opt.step()
    _agree(launches, opt, params)
    opt.state[params[1]][name].data = old.clone()          # the same tensor, its data elsewhere
    opt.step()
    _agree(launches, opt, params)


@pytest.mark.parametrize("bits", [32, 8])
def test_cleared_and_exchanged_states_begin_anew(launches, bits):
    params, opt = _made(bits)
    opt.step()
    kept = weakref.ref(opt.state[params[2]]["exp_avg"])
    opt.state.clear()
    gc.collect()
    assert kept() is None
    opt.step()
    assert set(opt.state) == set(params)
    _agree(launches, opt, params)
    opt.state[params[0]] = {k: v.clone() for k, v in opt.state[params[0]].items()}
    opt.step()
    _agree(launches, opt, params)


def test_other_bits_need_other_states(launches):
    for bits in (32, 8):
        params, opt = _made(bits)
        opt.step()
        opt.param_groups[0]["state_bits"] = 40 - bits
        launches.records = []
        with pytest.raises(ValueError):
            opt.step()
        assert not launches.records
        opt.state.clear()
        opt.step()
        _agree(launches, opt, params)


def test_a_master_that_is_asked_for_later(launches):
    params, opt = _made(32, False, torch.bfloat16)
    opt.step()
    opt.param_groups[0]["master"] = True
    opt.step()
    _agree(launches, opt, params)
    assert all(torch.equal(opt.state[p]["master"], p.detach().float()) for p in params)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("spoil", [lambda t: t[:-1].clone(), lambda t: t.to(torch.float16), lambda t: torch.stack((t, t), 1)[:, 0], lambda t: None,
                                   lambda t: torch.cat((t, t))])
def test_states_that_do_not_fit_are_refused(launches, bits, spoil):
    for name in ("exp_avg", "exp_avg_sq") if bits == 32 else ("exp_avg", "exp_avg_sqrt", "exp_avg_scale", "exp_avg_sqrt_scale"):
        params, opt = _made(bits)
        opt.step()
        t = opt.state[params[0]][name].flatten()
        if t.dtype == torch.float8_e4m3fn:
            spoiled = spoil(t.view(torch.uint8))
            spoiled = spoiled.view(torch.float8_e4m3fn) if spoiled is not None and spoiled.dtype == torch.uint8 else spoiled
        else:
            spoiled = spoil(t)
        opt.state[params[0]][name] = spoiled
        launches.records = []
        with pytest.raises(ValueError):
            opt.step()
        assert not launches.records


def test_loaded_states_are_taken_in_their_order(launches):
    params, opt = _made()
    opt.step()
    saved = opt.state_dict()
    turned = torch.arange(900.0).view(3, 300).t()
    saved["state"][0] = dict(saved["state"][0], exp_avg=turned)
    opt.load_state_dict(saved)
    opt.step()
    _agree(launches, opt, params)
    assert opt.state[params[0]]["exp_avg"].is_contiguous() and torch.equal(opt.state[params[0]]["exp_avg"], turned)
    saved["state"][0]["exp_avg"] = torch.zeros(899)        # of another model
    opt.load_state_dict(saved)
    launches.records = []
    with pytest.raises(ValueError):
        opt.step()
    assert not launches.records


def test_gradients_are_not_kept(launches):
    params, opt = _made()
    opt.step()
    refs = [weakref.ref(p.grad) for p in params]
    opt.zero_grad(set_to_none=True)
    gc.collect()
    assert all(r() is None for r in refs)
    turned = torch.ones(3, 300).t()
    opt.step(grads=[turned, torch.ones(256), torch.ones(7)])
    assert launches.records[0].grad != turned.data_ptr()   # a copy in the parameter's order
    ref = weakref.ref(turned)
    del turned
    gc.collect()
    assert ref() is None


def test_gradients_whose_data_is_exchanged(launches):
    params, opt = _made(dtype=torch.bfloat16)
    opt.step()
    for exchanged in (torch.ones(300, 3), torch.full((300, 3), 2.0, dtype=torch.bfloat16)):
        params[0].grad.data = exchanged
        opt.step()
        _agree(launches, opt, params)
    for bad in (torch.ones(300, 3, dtype=torch.float16), torch.ones(299, 3), torch.ones(3, 300)):
        params[0].grad.data = bad
        launches.records = []
        with pytest.raises(ValueError):
            opt.step()
        assert not launches.records


def test_parameters_whose_data_is_exchanged(launches):
    params, opt = _made()
    opt.step()
    params[0].data = params[0].data.clone()
    opt.step()
    _agree(launches, opt, params)
    params[0].data = params[0].data.to(torch.bfloat16)
    params[0].grad = torch.ones_like(params[0])
    opt.step()
    _agree(launches, opt, params)
    square = torch.nn.Parameter(torch.randn(8, 8))
    opt = asi.AdamW([square])
    square.grad = torch.ones(8, 8)
    opt.step()
    square.data = square.data.t()                          # the same address, another order
    with pytest.raises(TypeError):
        opt.step()


def test_a_tensor_on_another_device_is_refused(launches):
    params, opt = _made()
    opt.step()
    launches.records = []
    with pytest.raises(ValueError):
        opt.step(grads=[params[0].grad, torch.empty(256, device="meta"), params[2].grad])
    opt.state[params[1]]["exp_avg"] = torch.empty(256, device="meta")
    with pytest.raises(ValueError):
        opt.step()
    assert not launches.records


def test_gradients_given_for_the_parameters(launches):
    params, opt = _made(dtype=torch.bfloat16)
    grads = [torch.ones(p.shape) for p in params]
    opt.step(grads=tuple(grads))
    assert [r.grad for r in launches.records] == [g.data_ptr() for g in grads] and all(r.grad_dtype == B.ASI_F32 for r in launches.records)
    opt.step(grads=[None, grads[1], None])
    assert [r.grad for r in launches.records] == [grads[1].data_ptr()]
    for bad in (torch.ones(3, 300), torch.ones(300, 3, dtype=torch.float64), torch.ones(300, 3).to_sparse(), torch.ones(2, 3)):
        with pytest.raises(ValueError):
            opt.step(grads=[bad, *grads[1:]])


def test_lists_and_states_that_a_hash_changes():
    """A parameter's hash is Python code: what it changes is not read any more."""
    class Sly(torch.Tensor):
        act = None

        def __hash__(self):
            if Sly.act:
                Sly.act()
            return id(self)

    def inputs():
        params = [torch.Tensor._make_subclass(Sly, torch.zeros(50)) for _ in range(3)]
        states = {p: {"exp_avg": torch.zeros(50), "exp_avg_sq": torch.zeros(50)} for p in params}
        return params, [torch.zeros(50) for _ in params], states

    params, grads, states = inputs()
    made = B.adamw_records(params, grads, states, False, False, -1, 0.1, 0.0)
    records = (B.AdamwTensor * 3).from_buffer_copy(made)
    assert [r.exp_avg for r in records] == [states[p]["exp_avg"].data_ptr() for p in params]
    kept = list(params)
    for act in (lambda: params.clear(), lambda: grads.clear(), lambda: params.append(kept[0]), lambda: states.clear(), lambda: states.popitem() if states else None):
        Sly.act = None
        params, grads, states = inputs()
        kept = list(params)
        Sly.act = act
        assert B.adamw_records(params, grads, states, False, False, -1, 0.1, 0.0) is None
        Sly.act = None
