"""CPU: the build's commands, with a stand-in for the compiler that writes its
arguments down."""
import os
import stat
import sys

import pytest

from paper_2110_04175_amd import build


@pytest.fixture()
def commands(tmp_path, monkeypatch):
    log = tmp_path / "log"
    cc = tmp_path / "cc"
    cc.write_text(f"#!{sys.executable}\nimport sys\n"
                  f"open({str(log)!r}, 'a').write(' '.join(sys.argv[1:]) + '\\n')\n"
                  "out = sys.argv[sys.argv.index('-o') + 1]\n"
                  "open(out, 'w').close()\n"
                  "sys.exit(1 if '--fail' in sys.argv and '-c' in sys.argv else 0)\n")
    cc.chmod(cc.stat().st_mode | stat.S_IXUSR)
    sources = [str(tmp_path / "a.hip"), str(tmp_path / "b.hip")]
    monkeypatch.setattr(build, "HIPCC", str(cc))
    monkeypatch.setattr(build, "SOURCES", sources)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))

    def run(extra):
        build.build(extra=extra)
        return [line.split() for line in log.read_text().splitlines()]

    return run


def test_options_reach_every_step(commands):
    """Sanitizers and libraries are wanted by the link as well, libraries
    behind what needs them."""
    ran = commands(["--coverage", "-lm"])
    compiles, links = [c for c in ran if "-c" in c], [c for c in ran if "-c" not in c]
    assert len(compiles) == 2 and len(links) == 1
    for c in ran:
        assert "--coverage" in c and "-lm" in c and "--offload-arch=gfx950" in c
    link = links[0]
    assert "-shared" in link and link.index("-lm") > max(i for i, a in enumerate(link) if a.endswith(".o"))
    assert os.path.exists(build.LIB)


def test_a_source_that_does_not_compile_ends_the_build(commands):
    with pytest.raises(Exception):
        commands(["--fail"])
    assert not os.path.exists(build.LIB)
