"""The library needs neither torch's headers nor the host compiler: it is linked whatever becomes of the binding.  CPU only, nothing is compiled."""

import pytest

from paper_2403_11204_amd import build


def test_the_library_is_linked_where_the_binding_does_not_compile(monkeypatch):
    ran = []

    def no_headers(verbose):
        raise RuntimeError("g++ on binding.cpp failed")

    monkeypatch.setattr(build, "_compile", lambda unit, extra, verbose: unit)
    monkeypatch.setattr(build, "_compile_binding", no_headers)
    monkeypatch.setattr(build, "_run", lambda cmd, what, verbose: ran.append(cmd))
    with pytest.raises(RuntimeError, match="binding.cpp"):
        build.build(verbose=False)
    assert len(ran) == 1 and ran[0][ran[0].index("-o") + 1] == build.OUT and all(u in ran[0] for u in build.UNITS)
