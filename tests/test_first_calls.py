"""Bindings that fetch torch's types at their first call: two threads that make it at once, and every call after theirs."""
import builtins
import threading

import pytest

from paper_2605_05219_amd import block as BL, linear as LN, moe as MO


def no_tokens(name):
    import torch
    on = "cuda" if torch.cuda.is_available() else "cpu"
    bf = lambda *n: torch.zeros(*n, dtype=torch.bfloat16, device=on)  # noqa: E731
    if name == "moe":
        shape = MO.make_moe_shape(8, 2, 128, 64)
        return lambda: MO.gdn_moe(shape, bf(0, 128), bf(8, 128), torch.zeros(8, device=on), bf(8, 128, 128), bf(8, 128, 64), None, bf(0, 128),
                                  torch.zeros(0, 2, dtype=torch.int32, device=on), torch.zeros(0, 2, device=on), None)
    if name == "block":
        shape = BL.make_block_shape(64)
        return lambda: BL.gdn_block_norm(shape, bf(0, 64), None, None, None, None, torch.ones(64, device=on), None, None, bf(0, 64))
    return lambda: LN.gdn_linear_act(bf(0, 64), bf(8, 64), None, bf(0, 8), "silu")


@pytest.mark.parametrize("name,module,held", [("moe", MO, "_types"), ("block", BL, "_types"), ("linear", LN, "_codes")])
def test_two_first_calls_at_once(monkeypatch, name, module, held):
    call = no_tokens(name)
    call()
    of_a_call = getattr(module, held)
    monkeypatch.setattr(module, held, type(of_a_call)())
    meet, here, failed, real = threading.Barrier(2), threading.local(), [], builtins.__import__

    def slow_import(what, *args, **kw):
        if what == "torch" and getattr(here, "waits", False):            # both have seen that the types are not there
            here.waits = False
            meet.wait(timeout=30)
        return real(what, *args, **kw)

    def first():
        here.waits = True
        try:
            call()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    monkeypatch.setattr(builtins, "__import__", slow_import)
    threads = [threading.Thread(target=first) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    monkeypatch.setattr(builtins, "__import__", real)
    assert not failed
    call()
    assert getattr(module, held) == of_a_call
