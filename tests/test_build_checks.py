"""What the build looks at besides the compiler's exit status."""
import pytest

from paper_2505_24179_amd import build


def _compiler(tmp_path, monkeypatch, remarks):
    """In the place of hipcc: makes its output file and prints these remarks."""
    script = tmp_path / "hipcc"
    lines = "\n".join(f"d.hip:1:1: remark:     {r} [{build._REPORT}]" for r in remarks)
    script.write_text(f"#!/bin/sh\nfor last; do :; done\ntouch \"$last\"\ncat >&2 <<'END'\n{lines}\nEND\n")
    script.chmod(0o755)
    monkeypatch.setattr(build, "HIPCC", str(script))
    monkeypatch.setattr(build, "CSRC", str(tmp_path))


@pytest.mark.parametrize("remarks,sound", [(["Function Name: a", "ScratchSize [bytes/lane]: 0", "ScratchSize [bytes/lane]: 0"], True),
                                           (["ScratchSize [bytes/lane]: 0", "ScratchSize [bytes/lane]: 132"], False),
                                           (["ScratchSize [bytes/lane]: Unknown"], False), (["Function Name: a"], False), ([], False)])
def test_no_kernel_of_decode_is_built_with_scratch_memory(tmp_path, monkeypatch, remarks, sound):
    _compiler(tmp_path, monkeypatch, remarks)
    if sound:
        assert build._compile("decode.hip", []) == str(tmp_path / "decode.o") and (tmp_path / "decode.o").exists()
    else:
        with pytest.raises(RuntimeError, match="scratch"):
            build._compile("decode.hip", [])
        assert not (tmp_path / "decode.o").exists()
    assert build._compile("cache.hip", []) == str(tmp_path / "cache.o")


def test_decode_is_among_those_that_are_looked_at():
    assert set(build.NO_SCRATCH) <= set(build.SOURCES) and "decode.hip" in build.NO_SCRATCH
