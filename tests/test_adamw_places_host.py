"""AdamW's binding works with addresses that it takes once: the memory behind them stays theirs, and a step whose parameters have moved is refused before
the library is called (on the CPU, where a call that comes so far is refused for its device)."""
import gc

import pytest


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


def made(b, torch, eight=False):
    p, g = [torch.zeros(300), torch.zeros(0), torch.zeros(8, 4)], [torch.zeros(300), torch.zeros(0), torch.zeros(8, 4)]
    state = [[torch.zeros_like(t, dtype=torch.uint8 if eight else torch.float32) for t in p] for _ in range(2)]
    scales = [[torch.zeros(-(-t.numel() // 256)) for t in p] for _ in range(2)] if eight else [None, None]
    shadows = [t.bfloat16() for t in p]
    return b.AdamW(p, g, *state, *scales, shadows=shadows), {"param": p, "grad": g, "m": state[0], "v": state[1], "m_scale": scales[0], "v_scale": scales[1], "shadow": shadows}


def test_a_parameter_that_has_moved_is_refused():
    import torch
    b = sb()
    opt, tensors = made(b, torch)
    with pytest.raises(b.SBError, match="CUDA device"):          # (nothing has moved)
        opt.step(1e-3)
    p = tensors["param"][2]
    old = p.data                                                  # (alive, so that its address is not given away)
    p.data = torch.ones_like(p)
    for call in (lambda: opt.step(1e-3), opt.moments):
        with pytest.raises(b.SBError, match="moved"):
            call()
    p.data = old
    with pytest.raises(b.SBError, match="CUDA device"):
        opt.step(1e-3)
    tensors["param"][0].untyped_storage().resize_(0)
    with pytest.raises(b.SBError, match="moved"):
        opt.step(1e-3)


@pytest.mark.parametrize("eight", [False, True])
def test_the_memory_of_tensors_given_other_data_is_kept(eight):
    import torch
    from torch.multiprocessing.reductions import StorageWeakRef
    b = sb()
    opt, tensors = made(b, torch, eight)
    held = {}
    for name, ts in tensors.items():
        if ts is not None:
            held[name] = StorageWeakRef(ts[2].untyped_storage())
            ts[2].data = torch.ones_like(ts[2])
    gc.collect()
    assert not [name for name, ref in held.items() if ref.expired()]
    # gradients: until they are replaced
    opt.set_grads([torch.ones_like(t) for t in tensors["grad"]])
    gc.collect()
    assert held["grad"].expired() and not held["m"].expired()
