"""The binding's first call on tensors, from any number of host threads at once (no GPU: the call is refused for its tensor)."""
import dis
import threading

from paper_2608_18183_b200 import binding


def test_types_are_known_before_torch_is():
    """Whoever finds torch set goes on to look up types: the instruction that sets it is the last."""
    stores = [i.argval for i in dis.get_instructions(binding._rows) if i.opname == "STORE_GLOBAL"]
    assert stores == ["_types", "_torch"]


def test_first_calls_of_many_threads(monkeypatch):
    import torch
    x, said = torch.zeros(2, 8), []
    for _ in range(50):
        monkeypatch.setattr(binding, "_torch", None)
        monkeypatch.setattr(binding, "_types", {})

        def work():
            try:
                binding.hbsjd_distill(x, x)
            except binding.HbsjdError as e:
                said.append("not a tensor on a GPU" in str(e))

        threads = [threading.Thread(target=work) for _ in range(8)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    assert len(said) == 400 and all(said)
