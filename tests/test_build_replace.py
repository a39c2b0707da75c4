"""The build replaces the library file; it never writes into one that a running process may have mapped."""
import os
import subprocess
import tempfile

import pytest

from paper_1906_03707_b200 import build


@pytest.fixture
def library(tmp_path, monkeypatch):
    """A library file, a compiler that only writes its output, and a temporary folder on another file system if there is one."""
    lib, nvcc = tmp_path / "lib.so", tmp_path / "nvcc"
    lib.write_bytes(b"old")
    nvcc.write_text('#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\nprintf new > "$2"\n')
    nvcc.chmod(0o755)
    monkeypatch.setenv("NVCC", str(nvcc))
    monkeypatch.setattr(build, "LIB", str(lib))
    if os.path.isdir("/dev/shm") and os.access("/dev/shm", os.W_OK):
        monkeypatch.setattr(tempfile, "tempdir", "/dev/shm")
    return lib


def test_a_library_in_use_keeps_its_bytes(library):
    with open(library, "rb") as used:
        assert build.build(force=True) == str(library)
        assert used.read() == b"old" and library.read_bytes() == b"new"
    assert sorted(os.listdir(library.parent)) == ["lib.so", "nvcc"]


def test_a_failed_build_leaves_the_library(library):
    nvcc = library.parent / "nvcc"
    nvcc.write_text('#!/bin/sh\nfor a in "$@"; do [ "$a" = -shared ] && exit 1; done\nwhile [ "$1" != -o ]; do shift; done\nprintf new > "$2"\n')
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)
    assert library.read_bytes() == b"old" and sorted(os.listdir(library.parent)) == ["lib.so", "nvcc"]
