"""How the sources are compiled: each by itself, side by side, then linked."""
import subprocess

import pytest


@pytest.mark.parametrize("jobs", [None, "", "0", "3"])
def test_every_source_is_compiled_whatever_max_jobs_says(monkeypatch, jobs):
    from paper_2507_14668_amd import build
    ran = []
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: ran.append(cmd) or subprocess.CompletedProcess(cmd, 0, "", ""))
    monkeypatch.delenv("MAX_JOBS", raising=False)
    if jobs is not None:
        monkeypatch.setenv("MAX_JOBS", jobs)
    assert build.build() == build.LIB
    assert sorted(cmd[cmd.index("-c") + 1] for cmd in ran if "-c" in cmd) == build.sources()
    assert "-shared" in ran[-1] and build.LIB in ran[-1] and all("-shared" not in cmd for cmd in ran[:-1])
