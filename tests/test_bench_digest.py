"""What a traffic figure on record is tied to: the sources of the step's kernels, and no others."""
import os
import shutil

import pytest

import bench


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A copy of the sources that the digest is taken of."""
    for d in (os.path.join("paper_1906_00091_amd", "csrc"), "include"):
        shutil.copytree(os.path.join(bench.ROOT, d), tmp_path / d)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path


def append(tree, f, text="\n// more\n"):
    with open(tree / f, "a") as x:
        x.write(text)


@pytest.mark.parametrize("f", ["qk_rope.hip", "seq_attn.h", "seq_attn.hip", "seq_attn_f16.hip", "cache_attn.hip", "heads.h"])
def test_operators_over_histories_are_not_the_steps(tree, f):
    before = bench.source_digest()
    append(tree, "paper_1906_00091_amd/csrc/" + f)
    assert bench.source_digest() == before
    p = tree / "include" / "dlrm_hot.h"
    p.write_text(p.read_text().replace("int32_t dlrm_cache_attn(", "int32_t dlrm_cache_attention("))
    assert bench.source_digest() == before


@pytest.mark.parametrize("f", ["bwd_reduce.h", "bwd_reduce_sgd.hip", "common.h", "emb_fwd.hip", "interact.hip", "pooled_interact.hip", "bwd_sort.h"])
def test_the_steps_own_sources_are(tree, f):
    before = bench.source_digest()
    append(tree, "paper_1906_00091_amd/csrc/" + f)
    assert bench.source_digest() != before


def test_the_steps_part_of_the_public_header_is(tree):
    before = bench.source_digest()
    p = tree / "include" / "dlrm_hot.h"
    p.write_text(p.read_text().replace("int32_t dlrm_emb_bag_fwd(", "int32_t dlrm_emb_bag_forward("))
    assert bench.source_digest() != before
