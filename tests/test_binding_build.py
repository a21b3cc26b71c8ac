"""The torch module of the store calls is built anew for another torch, and a stale one is refused (no GPU needed)."""
import pytest
import torch

import paper_2512_00504_b200 as gkv


class Built(Exception):
    pass


def test_another_torch_needs_another_build(monkeypatch):
    path = gkv.build_binding()
    monkeypatch.setattr(gkv.subprocess, "check_call", lambda cmd: (_ for _ in ()).throw(Built(cmd)))
    assert gkv.build_binding() == path                 # nothing has changed: nothing is built
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "9.9.9")
        with pytest.raises(Built) as e:
            gkv.build_binding()
        assert any("9.9.9" in str(a) for a in e.value.args[0])
        m.setattr(gkv, "_binding", None)
        with pytest.raises(RuntimeError, match="9.9.9"):
            gkv._torch_binding()
    gkv._torch_binding()
