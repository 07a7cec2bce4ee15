"""Host-only: the package's names are the binding's, now and after the binding has been changed (a wrapper for tracing, a test's replacement)."""
import importlib
from unittest import mock

import paper_1812_07625_amd as P
from paper_1812_07625_amd import binding

NAMES = ("w2l_version", "w2l_distill_launch_config", "w2l_ctc_fwd_bwd", "workspace")


def test_a_replaced_entry_point_is_seen_through_the_package(monkeypatch):
    for name in NAMES:
        before = getattr(P, name)
        assert before is getattr(binding, name)
        with monkeypatch.context() as m:
            m.setattr(binding, name, lambda *a: "replaced")
            assert getattr(P, name)() == "replaced", name
        assert getattr(P, name) is before
        with mock.patch.object(binding, name) as m:
            assert getattr(P, name) is m
        assert getattr(P, name) is before


def test_an_entry_point_replaced_in_the_package_stays_so():
    """What a program puts on the package itself is its own, whatever happens to the binding."""
    before = P.w2l_version
    with mock.patch.object(P, "w2l_version") as m:
        binding.w2l_version = binding.w2l_version
        assert P.w2l_version is m
    assert P.w2l_version is before


def test_removed_and_added_names():
    binding.w2l_more = lambda: 7
    assert P.w2l_more() == 7 and P.w2l_more() == 7
    del binding.w2l_more
    assert not hasattr(P, "w2l_more")


def test_a_binding_that_is_loaded_again():
    before = [getattr(P, n) for n in NAMES]
    kept = dict(binding.__dict__)
    try:
        importlib.reload(binding)
        assert all(getattr(P, n) is getattr(binding, n) and getattr(P, n) is not b for n, b in zip(NAMES, before))
    finally:
        for n, v in kept.items():
            if not n.startswith("__"):
                setattr(binding, n, v)
    assert [getattr(P, n) for n in NAMES] == before
