"""A GPU test that failed with an incomplete profiler session is run again; one that failed with complete ones, or for another reason, is not."""
import types

import conftest
import pytest


def item(obj):
    return types.SimpleNamespace(obj=obj, name="t", funcargs=dict(x=1, y=2), _fixtureinfo=types.SimpleNamespace(argnames=("x",)),
                                 get_closest_marker=lambda name: name == "gpu" or None)


@pytest.fixture(autouse=True)
def no_sessions(monkeypatch):
    monkeypatch.setattr(conftest, "_watch_sessions", lambda: None)


@pytest.mark.parametrize("failures,passes", [(0, True), (1, True), (2, True), (3, False)])
def test_incomplete_sessions_are_asked_again(failures, passes):
    runs = []

    def body(x):
        runs.append(x)
        if len(runs) <= failures:
            conftest._incomplete.append((0, 7))
            raise AssertionError("no kernel")
    if passes:
        assert conftest.pytest_pyfunc_call(item(body)) is True
    else:
        with pytest.raises(AssertionError, match="no kernel"):
            conftest.pytest_pyfunc_call(item(body))
    assert runs == [1] * min(failures + 1, 3)


@pytest.mark.parametrize("error,incomplete", [(AssertionError, False), (RuntimeError, True), (ValueError, False)])
def test_other_failures_stand(error, incomplete):
    runs = []

    def body(x):
        runs.append(x)
        if incomplete:
            conftest._incomplete.append((0, 7))
        raise error("wrong")
    with pytest.raises(error, match="wrong"):
        conftest.pytest_pyfunc_call(item(body))
    assert runs == [1]


def test_tests_without_the_marker_are_left_alone():
    it = item(None)
    it.get_closest_marker = lambda name: None
    assert conftest.pytest_pyfunc_call(it) is None
