"""The graph-transformer operators' kernels for whole-vector rows keep every value in
registers: compiled for gfx950, they use no per-lane scratch memory. Named beside each
source: kernels that may not spill, as they appear in the mangled symbols; the others are
forms for odd widths or huge bias tables, and the one over small graphs of bf16 heads of 16
columns with a bias, whose few spilled registers buy a third wavefront a SIMD."""

import re

import pytest

from test_no_spills import _resource_usage

HOT = {
    "embed.hip": ["embed"],
    "group_norm.hip": ["norm_waves", "norm_sums", "norm_apply"],
    "attention_bf16_narrow.hip": [r"attn_fwd.*Li8E", "attn_small"],
    "attention_f32_narrow.hip": [r"attn_fwd.*Li8E", "attn_small"],
    "attention_grad_bf16_narrow.hip": [r"attn_grad_q.*Li4ELi\dELi8E", r"attn_grad_kv.*Li4ELi\dELi8E"],
    "attention_grad_bf16_wide.hip": [r"attn_grad_q.*Li4ELi\dELi8E", r"attn_grad_kv.*Li4ELi\dELi8E"],
}


@pytest.mark.parametrize("src", sorted(HOT))
def test_hot_kernels_do_not_spill(src):
    usage = _resource_usage(src)
    for pattern in HOT[src]:
        found = [sym for sym in usage if re.search(pattern, sym)]
        assert found, f"no kernel {pattern} in {src}"
        for sym in found:
            scratch = usage[sym].get("ScratchSize", 0)
            assert scratch == 0, f"{sym}: {scratch} bytes/lane of scratch"
