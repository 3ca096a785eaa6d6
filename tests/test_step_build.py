"""The compiled part of the binding goes with the torch and the Python that it was built against."""
import os
import types

import pytest

from paper_2506_09397_b200 import binding as B
from paper_2506_09397_b200 import build as builder


def test_the_marshalling_is_built_again_for_another_torch(tmp_path, monkeypatch):
    built = []

    def run(cmd):
        built.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w"):
            pass

    monkeypatch.setattr(builder, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(builder, "OBJ", str(tmp_path))
    builder.build_marshal(False, run)
    builder.build_marshal(False, run)
    assert len(built) == 1 and os.path.exists(builder.MARSHAL)
    monkeypatch.setattr(builder, "version", lambda name: "1.0.0+other")
    builder.build_marshal(False, run)
    builder.build_marshal(False, run)
    assert len(built) == 2 and any("1.0.0+other" in x for x in built[1])
    builder.build_marshal(True, run)
    assert len(built) == 3


def test_the_marshalling_of_another_torch_is_not_used(monkeypatch):
    builder.build()
    assert B.marshal().built_for == builder.marshal_for()
    monkeypatch.setattr(B, "_marshal", None)
    monkeypatch.setattr(builder, "version", lambda name: "1.0.0+other")
    with pytest.raises(RuntimeError, match="1.0.0.other"):
        B.marshal()
    monkeypatch.undo()
    assert isinstance(B.marshal(), types.ModuleType)
