"""What compiles the library is what its digests name: the environment adds nothing to the compiler's flags."""
import subprocess

from paper_2509_03047_gb300 import build


def test_the_environment_adds_no_compiler_flags(monkeypatch, tmp_path):
    def commands(name):
        made = []

        def run(cmd, **kw):
            made.append([a.replace(str(tmp_path / name), "") for a in cmd])
            open(cmd[cmd.index("-o") + 1], "w").close()
            return subprocess.CompletedProcess(cmd, 0, "", "")

        monkeypatch.setattr(build, "OUT_DIR", str(tmp_path / name))
        monkeypatch.setattr(build, "LIB", str(tmp_path / name / "lib.so"))
        monkeypatch.setattr(build.subprocess, "run", run)
        build.build(force=True)
        return sorted(made)

    plain = commands("plain")
    assert len(plain) == len(build.SOURCES) + 1
    for name in ("FR_EXTRA", "NVCC_FLAGS", "NVCCFLAGS", "CXXFLAGS", "CFLAGS"):
        monkeypatch.setenv(name, "-DFR_FROM_THE_ENVIRONMENT -use_fast_math")
    assert commands("set") == plain
    for cmd in plain:
        assert set(build.ARCH) <= set(cmd) and ("-c" not in cmd or set(build.NVCC_FLAGS) <= set(cmd))
