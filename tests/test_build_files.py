"""Which files a build reads and writes."""
import pytest


def test_a_missing_library_of_the_memory_is_built_beside_the_one_that_is_there(monkeypatch, tmp_path):
    """libbps.so may be loaded: with another one in its place the memory's library would load that one too, and tell its failures to it."""
    from paper_2103_07013_amd import build, memory
    made = []

    def note(libs, verbose):
        made.extend(lib for _, lib, _ in libs)
        raise RuntimeError("nothing is built here")

    monkeypatch.setattr(build, "_make", note)
    monkeypatch.setattr(build, "MEMORY_LIB", str(tmp_path / "libbps_memory.so"))
    monkeypatch.setattr(memory, "_lib", None)
    with pytest.raises(RuntimeError, match="nothing is built here"):
        memory._library()
    assert made == [build.MEMORY_LIB]


def test_a_build_makes_both_libraries(monkeypatch):
    from paper_2103_07013_amd import build
    made = []
    monkeypatch.setattr(build, "_make", lambda libs, verbose: made.extend(libs))
    assert build.build() == build.LIB
    assert [lib for _, lib, _ in made] == [build.LIB, build.MEMORY_LIB] and made[0][0] == build.SOURCES and made[1][0] == build.MEMORY_SOURCES


def test_sources_are_named_as_from_the_working_folder(monkeypatch, tmp_path):
    from paper_2103_07013_amd import build
    monkeypatch.chdir(tmp_path)
    (tmp_path / "k.cpp").write_text('extern "C" int answer(void) { return 42; }\n')
    build.compile_hip(["k.cpp"], "k.so")
    import ctypes
    assert ctypes.CDLL(str(tmp_path / "k.so")).answer() == 42
