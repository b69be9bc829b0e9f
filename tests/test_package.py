"""The package's names are the binding's, also after one of them is rebound there."""
import os
import subprocess
import sys

import pytest


@pytest.fixture(scope="module")
def rr():
    import paper_2402_12399_b200 as package
    from paper_2402_12399_b200 import build
    build.build()
    return package


def test_a_rebound_name_of_the_binding_is_seen_through_the_package(rr, monkeypatch):
    before = rr.check, rr.linear_fwd, rr.BF16                        # (a first look must not keep what it found)
    monkeypatch.setattr(rr.binding, "check", "a wrapper")
    monkeypatch.setattr(rr.binding, "linear_fwd", "another")
    assert rr.check == "a wrapper" and rr.linear_fwd == "another"
    monkeypatch.undo()
    assert (rr.check, rr.linear_fwd, rr.BF16) == before


def test_every_public_name_is_there(rr):
    import paper_2402_12399_b200.binding as binding
    for name in rr._BINDING:
        assert getattr(rr, name) is getattr(binding, name), name
    assert rr.binding is binding
    with pytest.raises(AttributeError):
        rr.no_such_name


def test_a_binding_imported_and_patched_before_the_first_look():
    code = ("import paper_2402_12399_b200.binding as b\nimport paper_2402_12399_b200 as rr\nb.route = 1\nassert rr.route == 1\nb.route = 2\nassert rr.route == 2\n"
            "del b.route\ntry:\n    rr.route\n    raise SystemExit('kept a deleted name')\nexcept AttributeError:\n    pass\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True).returncode == 0
