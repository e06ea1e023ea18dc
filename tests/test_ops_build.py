"""When the operators' binding is built: with torch, and again for another torch."""
import os

import pytest


@pytest.fixture()
def B():
    from paper_2609_27193_gb300 import build
    build.build()
    return build


def test_another_torch_makes_it_stale(B, monkeypatch):
    if B.binding_for() is None:
        pytest.skip("no torch")
    assert B.binding_up_to_date()
    monkeypatch.setattr(B, "binding_for", lambda: "torch 0.0 at nowhere, none")
    assert not B.binding_up_to_date()


def test_the_library_builds_without_torch(B, monkeypatch):
    find = B.importlib.util.find_spec
    monkeypatch.setattr(B.importlib.util, "find_spec", lambda name: None if name == "torch" else find(name))
    monkeypatch.setattr(B, "compile_binding", lambda: pytest.fail("compiled the binding without torch"))
    monkeypatch.setattr(B, "link_binding", lambda *a: pytest.fail("linked the binding without torch"))
    monkeypatch.setattr(B, "build_library", lambda *a: B.LIB)
    assert B.binding_for() is None
    assert B.build() == B.LIB and B.build(force=True) == B.LIB
    assert os.path.exists(B.LIB)
