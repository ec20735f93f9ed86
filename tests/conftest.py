import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


# Tests that name the kernels which ran take them from a profiler session.  Sessions come back without the device's records of their first
# launches now and then (as many as all of them), whatever was launched; such a session says nothing about the kernels.  A test that failed
# with one is run again, up to twice; a session with a kernel for every launch is taken at its word.
_incomplete = []


def _watch_sessions():
    import torch
    leave = torch.profiler.profile.__exit__
    if getattr(leave, "watched", False):
        return

    def watched(self, *args):
        done = leave(self, *args)
        names = [e.name for e in self.events() or ()]
        launches = sum(n in ("hipLaunchKernel", "hipExtLaunchKernel", "hipModuleLaunchKernel", "hipExtModuleLaunchKernel") for n in names)
        kernels = sum(not n.startswith(("hip", "Memcpy", "Memset")) for n in names)
        if kernels < launches or not names:
            _incomplete.append((kernels, launches))
        return done

    watched.watched = True
    torch.profiler.profile.__exit__ = watched


@pytest.hookimpl(tryfirst=True)
def pytest_pyfunc_call(pyfuncitem):
    if pyfuncitem.get_closest_marker("gpu") is None:
        return None
    _watch_sessions()
    args = {name: pyfuncitem.funcargs[name] for name in pyfuncitem._fixtureinfo.argnames}
    for again in (True, True, False):
        _incomplete.clear()
        try:
            pyfuncitem.obj(**args)
            return True
        except AssertionError:
            if not again or not _incomplete:
                raise
            print(f"{pyfuncitem.name}: {_incomplete} kernels of launches in the profiler's sessions; once more", flush=True)


@pytest.fixture(scope="session")
def oracle_mod():
    import oracle
    oracle.build()
    return oracle
