"""The listing rules of test_ffn_codegen.py for the gated feed-forward block's tiles with fp32 factors."""
import os

import pytest

import paper_2505_23725_amd as mlc
import test_ffn_codegen as ffn
import test_gemm_codegen as rules

FORMS = [(5, 0), (5, 1), (6, 0)]          # both projections with either activation, the inner gradients
HAND = ["ffn_gemm_kernelILi%dELi%dELi256ELi256E" % f for f in FORMS]
SMALL = ["ffn_gemm_kernelILi%dELi%dELi%dELi128ELi%dE" % (*f, bm, ring) for f in FORMS for bm in (64, 128) for ring in (5, 9)]


@pytest.mark.skipif(not os.path.exists(rules.OBJDUMP), reason="no llvm-objdump")
def test_no_accumulator_is_read_early_and_resources_are_whole(tmp_path, monkeypatch):
    mlc.library()
    monkeypatch.setattr(rules, "KERNELS", HAND + SMALL)
    code = rules.listing(str(tmp_path))
    assert sorted(code) == sorted(HAND + SMALL)
    for name, forms in code.items():
        assert len(forms) == 1, name
        ins = forms[0]
        assert any(i.to_lds for i in ins), name
        if name in HAND:      # 128 MFMAs in a tile's first K tile, its plain ones and those at an end, 256 reads an epilogue
            assert (sum(i.mfma for i in ins), sum(i.op.startswith("v_accvgpr_read") for i in ins)) == (3 * 128, 256), name
        assert not rules.faults(ins, name in HAND), (name, rules.faults(ins, name in HAND)[:5])
        assert not any(i.op.startswith("scratch_") for i in ins), name
        assert not ffn.lost_resources(ins), (name, ffn.lost_resources(ins)[:4])
