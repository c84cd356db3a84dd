"""What the packed-sequence binding answers on the host; no GPU is needed."""
import ctypes as C

import pytest

from paper_2507_14959_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


@pytest.mark.parametrize("sizes", [
    dict(heads=5, kv_heads=5, head_dim=128, n_seqs=1, max_q=4096, max_kv=4096, workspace_bytes=1 << 28),
    dict(heads=6, kv_heads=2, head_dim=64, n_seqs=2, max_q=700, max_kv=9000, q_rows=793, kv_rows=9303, workspace_bytes=1 << 28),
    dict(heads=8, kv_heads=8, head_dim=64, n_seqs=4, max_q=300, max_kv=300), dict(heads=8, kv_heads=8, head_dim=64, n_seqs=16, max_q=100, max_kv=100)])
def test_the_kernel_of_a_call_is_told_for_its_own_order(lib, sizes):
    """Causal and full calls of these sizes take different forms; each is told as the library takes it."""
    told = []
    for causal in (True, False):
        s = dict(sizes)
        space = s.pop("workspace_bytes", 0)
        rows = {"q_rows": s["n_seqs"] * s["max_q"], "kv_rows": s["n_seqs"] * s["max_kv"], **s}
        width = {n: s[h] * s["head_dim"] for n, h in (("q_stride", "heads"), ("out_stride", "heads"), ("k_stride", "kv_heads"), ("v_stride", "kv_heads"))}
        some = {n: 1 << 20 for n in ("q", "k", "v", "out", "q_offsets", "kv_offsets")}
        args = binding.pm_packed_attention(**rows, **width, **some, causal=int(causal), workspace=(1 << 20) if space else None, workspace_bytes=space)
        form = (C.c_int32 * 3)()
        assert lib.pm_attention_packed_kernel(C.byref(args), 148, form) == 0
        told.append(binding.attention_packed_kernel(**sizes, causal=causal))
        assert told[-1] == (("16 rows", "tcgen05", "fp32")[form[0]], form[1], form[2])
    assert told[0] != told[1]


@pytest.mark.parametrize("scale,refused", [(2.3e38, False), (2.4e38, True), (3.4e38, True)])
def test_a_scale_whose_exponent_of_two_overflows_is_refused(lib, scale, refused):
    """Times log2(e) it would be infinite, and products that are zero would come out as no numbers."""
    some = {n: 1 << 20 for n in ("q", "k", "v", "out", "q_offsets")}
    args = binding.pm_packed_attention(**some, q_stride=128, k_stride=128, v_stride=128, out_stride=128, q_rows=8, kv_rows=8, n_seqs=1, max_q=8, max_kv=8,
                                       heads=2, kv_heads=2, head_dim=64, scale=scale)
    form = (C.c_int32 * 3)()
    assert lib.pm_attention_packed_kernel(C.byref(args), 148, form) == (binding.PM_ERR_ARG if refused else 0)
    if refused:
        assert lib.pm_attention_packed(C.byref(args), None) == binding.PM_ERR_ARG
