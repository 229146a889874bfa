"""What every HIP source is compiled with (paper_2406_09904_amd/build.py)."""
import types

from paper_2406_09904_amd import build


def test_every_source_is_compiled_without_what_the_compiler_gets_wrong(monkeypatch, tmp_path):
    """Packed fp32 instructions off, the execution mask restored at the end of every branch: not in some sources only."""
    commands = []

    def run(cmd, **more):
        commands.append(cmd)
        out = cmd[cmd.index("-o") + 1] if "-o" in cmd else None
        if out:
            open(out, "w").close()
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(build.subprocess, "run", run)
    build.build(out_dir=str(tmp_path))
    compiled = [c for c in commands if any(a.endswith(".hip") for a in c)]
    assert len(compiled) == len(build.SOURCES)
    for c in compiled:
        assert "-packed-fp32-ops" in c and "-amdgpu-remove-redundant-endcf=0" in c, [a for a in c if a.endswith(".hip")]
