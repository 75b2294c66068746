"""Which sources the hazard scan (tests/isa_check.py) looks at, and how closely.  CPU only."""
import os
import re

import pytest

from tests import isa_check


def text(f):
    """Without its comments."""
    return re.sub(r"//.*", "", open(os.path.join(isa_check.CSRC, f)).read())


def sources():
    return [f for f in sorted(os.listdir(isa_check.CSRC)) if f.endswith(".hip")]


@pytest.mark.parametrize("src", ["attn_extend_bf16.hip", "cache_weights.hip"])
def test_a_serving_step_is_scanned_on_straight_paths_too(src):
    """A tile of the 16 x 16 instruction that changes registers between two steps of a sum, or is read within eleven wait states, is a finding here."""
    assert src in isa_check.KERNEL_SOURCES and src not in isa_check.ASM_FREE_SOURCES
    hits = isa_check.scan(isa_check.assembly(src))
    assert not hits, hits


def test_every_matrix_instruction_of_any_size_is_scanned():
    for f in sources():
        if re.search(r"\bmfma\d+\w*(<\w+>)?\(|__builtin_amdgcn_(s|d)?mfma|v_s?mfma", text(f)):
            assert f in isa_check.KERNEL_SOURCES, f


def test_sources_scanned_across_branches_only_hold_no_matrix_instructions_in_assembly():
    for f in isa_check.ASM_FREE_SOURCES:
        assert not re.search(r"mfma\w*_vgpr|v_s?mfma", text(f)), f
