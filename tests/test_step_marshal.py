"""The binding's C part: built for this interpreter where that can be done, and not needed where it cannot (CPU)."""
import os
import sysconfig

import pytest
import torch

import paper_2310_12670_amd as reft
from paper_2310_12670_amd import build


def test_built_for_this_interpreter(tmp_path):
    assert build.MARSHAL.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    out = str(tmp_path / os.path.basename(build.MARSHAL))
    assert build.build_marshal(out) and os.path.getsize(out) > 0
    assert reft.binding._load_marshal().__file__ == build.MARSHAL


def test_a_machine_without_pythons_headers_builds_the_rest(tmp_path, monkeypatch):
    out = tmp_path / "m.so"
    out.write_bytes(b"of an earlier build")
    assert build.build_marshal(str(out), include=str(tmp_path)) is False and not out.exists()
    monkeypatch.setattr(build.shutil, "which", lambda name: None)
    assert build.build_marshal(str(out)) is False


def test_calls_without_it(monkeypatch):
    """The same checks, by the binding's Python part."""
    def missing(name, package):
        raise ModuleNotFoundError(name)
    monkeypatch.setattr(reft.binding, "_marshal", None)
    monkeypatch.setattr(reft.binding, "_TYPE_OF", {})
    monkeypatch.setattr(reft.binding.importlib, "import_module", missing)
    x = torch.zeros(4, 8)
    for y in (torch.zeros(4, 9), x.bfloat16(), x):                             # the last is right but for the memory
        with pytest.raises(reft.ReftError) as e:
            reft.reft_dropout(x, y, 0.1, 1)
        assert e.value.code == reft.REFT_EINVAL
    with pytest.raises(reft.ReftError) as e:
        wide = torch.zeros(1, 65537)
        reft.reft_norm_forward(wide, None, torch.ones(65537), 1e-5, y=wide)
    assert e.value.code == reft.REFT_ESIZE
    reft.reft_dropout(torch.zeros(0, 8), torch.zeros(0, 8), 0.1, 1)
