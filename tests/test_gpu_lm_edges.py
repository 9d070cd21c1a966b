"""The language-model operators (include/asi_lm.h) where they meet what is exchanged, removed, overwritten or extreme."""
import copy

import pytest
import torch

import paper_2505_05086_amd as asi

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(seed, *shape):
    return torch.empty(*shape, device="cuda").normal_(generator=_gen(seed))


# ---- AdamW: what is exchanged between steps --------------------------------------------------------------
def _drop_master(opt, p):
    with torch.no_grad():
        p.copy_(p.float() * 0.5)
    del opt.state[p]["master"]


def _replace(name):
    def change(opt, p):
        t = opt.state[p][name]
        opt.state[p][name] = torch.full_like(t, 0.25) if t.dtype == torch.float32 else t.view(torch.uint8).flip(0).contiguous().view(t.dtype)
    return change


def _exchange(name):
    def change(opt, p):
        opt.state[p][name].data = opt.state[p][name].data.clone()
    return change


@pytest.mark.parametrize("bits,change", [(32, _drop_master), (8, _drop_master), (32, _replace("exp_avg_sq")), (8, _replace("exp_avg_sqrt")),
                                         (8, _replace("exp_avg_sqrt_scale")), (32, _exchange("exp_avg_sq")), (8, _exchange("master")),
                                         (32, lambda opt, p: opt.state.clear()), (8, lambda opt, p: opt.state.clear()),
                                         (32, lambda opt, p: opt.state.__setitem__(p, {}))])
def test_adamw_goes_on_from_what_its_states_are(bits, change):
    """The step after a change is that of an optimiser that never had another state, bit for bit."""
    params = [torch.nn.Parameter(_randn(k, n).to(torch.bfloat16)) for k, n in enumerate((1000, 300))]
    opt = asi.AdamW(params, lr=1e-2, state_bits=bits, master=True)
    for k, p in enumerate(params):
        p.grad = _randn(10 + k, p.numel()).to(torch.bfloat16)
    opt.step()
    opt.step()
    change(opt, params[0])
    junk = torch.full((1 << 20,), NAN, device="cuda")        # over what was freed
    others = [torch.nn.Parameter(p.detach().clone()) for p in params]
    fresh = asi.AdamW(others, lr=1e-2, state_bits=bits, master=True)
    fresh.param_groups[0]["step"] = opt.param_groups[0]["step"]
    for p, q in zip(params, others):
        q.grad = p.grad.clone()
        if p in opt.state:
            fresh.state[q] = copy.deepcopy(dict(opt.state[p]))
    opt.step()
    fresh.step()
    assert torch.isnan(junk).all()
    for p, q in zip(params, others):
        assert torch.equal(p, q) and set(opt.state[p]) == set(fresh.state[q])
        for name, t in opt.state[p].items():
            assert torch.equal(t.view(torch.uint8), fresh.state[q][name].view(torch.uint8)), name


def test_adamw_refuses_a_tensor_that_left_its_gpu():
    params = [torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (100, 300)]
    opt = asi.AdamW(params)
    for p in params:
        p.grad = torch.ones_like(p)
    opt.step()
    before = params[0].detach().clone()
    opt.state[params[1]]["exp_avg"] = opt.state[params[1]]["exp_avg"].cpu()
    with pytest.raises(ValueError):
        opt.step()
    assert torch.equal(params[0], before)
