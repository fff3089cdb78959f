"""The kernels compute infinities and NaN on purpose (rows without keys, scores out
of range, a caller's own), so no source is compiled with a licence to take them
as absent."""
from paper_2608_03057_amd import build


def test_no_source_is_compiled_without_infinities_or_nans(monkeypatch):
    commands = []
    monkeypatch.setattr(build.subprocess, "check_call", commands.append)
    for src in build.SOURCES + build.PROBE_SOURCES:
        build._compile(src)
    assert len(commands) == len(build.SOURCES + build.PROBE_SOURCES)
    for cmd in commands:
        for flag in cmd:
            assert flag not in ("-ffast-math", "-Ofast", "-ffinite-math-only", "-fno-honor-nans",
                                "-fno-honor-infinities", "-menable-no-nans",
                                "-menable-no-infs"), cmd
