"""Which files a stored HBM reading belongs to: the kernel's source and what it includes, whatever the headers are called (no GPU)."""
import os

import pytest

from paper_2510_25979_amd import build, traffic


@pytest.fixture
def csrc(tmp_path, monkeypatch):
    monkeypatch.setattr(traffic, "HERE", str(tmp_path))
    os.mkdir(tmp_path / "csrc")
    files = {"apply.hip": '#include <hip/hip_runtime.h>\n#include "near.h"\n  #  include "tile.hpp"\n// #include "named.h"\n', "exact.hip": '#include "tile.hpp"\n',
             "near.h": '#pragma once\n#include "far.hpp"\n#include "near.h"\n', "far.hpp": '#include "../elsewhere.h"\n', "tile.hpp": "", "named.h": "", "other.hpp": ""}

    def write(name, text=None):
        (tmp_path / "csrc" / name).write_text(files[name] if text is None else text)

    for name in files:
        write(name)
    return write


def test_a_reading_belongs_to_the_source_and_all_it_includes(csrc):
    assert traffic.sources_of("apply_bf16_kernel") == ["apply.hip", "far.hpp", "near.h", "tile.hpp"]
    assert traffic.sources_of("exact_bf16_kernel") == ["exact.hip", "tile.hpp"]
    at = {k: traffic.source_revision(k) for k in ("apply_bf16_kernel", "exact_bf16_kernel")}
    for name, apply, exact in (("near.h", True, False), ("far.hpp", True, False), ("tile.hpp", True, True), ("apply.hip", True, False), ("exact.hip", False, True),
                               ("other.hpp", False, False), ("named.h", False, False)):
        csrc(name, open(os.path.join(traffic.HERE, "csrc", name)).read() + "// changed\n")
        assert (traffic.source_revision("apply_bf16_kernel") != at["apply_bf16_kernel"]) == apply, name
        assert (traffic.source_revision("exact_bf16_kernel") != at["exact_bf16_kernel"]) == exact, name
        csrc(name)
    assert at == {k: traffic.source_revision(k) for k in at}


def test_a_header_that_takes_another_name_counts(csrc):
    before = traffic.source_revision("exact_bf16_kernel")
    csrc("near.h", "")
    csrc("exact.hip", '#include "near.h"\n')
    assert traffic.sources_of("exact_bf16_kernel") == ["exact.hip", "near.h"] and traffic.source_revision("exact_bf16_kernel") != before


def test_every_header_is_some_kernels_and_the_build_knows_it():
    known = {h for h in build.HEADERS if "/" not in h}
    assert known == {n for n in os.listdir(build.CSRC) if n.endswith((".h", ".hpp"))}
    used = {n for s in build.SOURCES if s != "api.hip" for n in traffic.sources_of(s[:-4] + "_kernel")[1:]}
    assert used == known      # (launch.hpp and serve.h are api.hip's, too)
