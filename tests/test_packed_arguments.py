"""Refusals of the packed-sequence operators and what their binding passes on; no GPU is needed."""
import ctypes as C
import math

import pytest

from paper_2507_14959_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


ADDRESS = 1 << 20                    # aligned, never read: every call below is refused before a launch


def attention(**changes):
    v = dict(q=ADDRESS, k=ADDRESS, v=ADDRESS, out=ADDRESS, q_stride=256, k_stride=128, v_stride=128, out_stride=256, q_offsets=ADDRESS, q_rows=8, kv_rows=8,
             n_seqs=1, max_q=8, max_kv=8, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.0, dtype=0)
    v.update(changes)
    return binding.pm_packed_attention(**v)


@pytest.mark.parametrize("changes", [
    dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q_offsets=None), dict(q=ADDRESS + 8), dict(k=ADDRESS + 2), dict(out=ADDRESS + 4),
    dict(q_stride=255), dict(q_stride=260), dict(k_stride=64), dict(v_stride=132), dict(out_stride=0), dict(heads=3), dict(heads=0), dict(kv_heads=0),
    dict(head_dim=96), dict(head_dim=0), dict(q_rows=-1), dict(kv_rows=-1), dict(n_seqs=-1), dict(max_q=-1), dict(max_kv=-1), dict(dtype=2),
    dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(kv_lengths=ADDRESS)])
def test_attention_refuses(lib, changes):
    assert lib.pm_attention_packed(C.byref(attention(**changes)), None) == binding.PM_ERR_ARG


@pytest.mark.parametrize("changes", [dict(n_seqs=4097), dict(heads=130, kv_heads=2, q_stride=130 * 64, out_stride=130 * 64),
                                     dict(q_rows=1 << 30, max_q=1 << 30, heads=2, kv_heads=1)])
def test_attention_capacity(lib, changes):
    assert lib.pm_attention_packed(C.byref(attention(**changes)), None) == binding.PM_ERR_CAPACITY


def test_null_arguments(lib):
    assert lib.pm_attention_packed(None, None) == binding.PM_ERR_ARG
    assert lib.pm_qk_norm_rope(None, None) == binding.PM_ERR_ARG
    assert lib.pm_rope_init(None, None) == binding.PM_ERR_ARG
    assert lib.pm_rope(ADDRESS, 64, ADDRESS, 64, ADDRESS, 1, 1, None, 0, None) == binding.PM_ERR_ARG


@pytest.mark.parametrize("changes", [dict(head_dim=0), dict(head_dim=72), dict(rot_dim=8), dict(rot_dim=0), dict(rot_dim=128), dict(axes=3), dict(axes=0),
                                     dict(base=0.0), dict(base=-1.0), dict(base=math.inf), dict(base=math.nan), dict(amplitude=math.nan),
                                     dict(scaling="linear", factor=0.0), dict(scaling="ntk", factor=math.nan), dict(scaling="other"),
                                     dict(scaling="bands", factor=2.0, original=0.0), dict(scaling="bands", factor=2.0, original=10.0, low_turns=4.0),
                                     dict(base=1e-308, head_dim=256), dict(scaling="ntk", factor=1e308)])
def test_rope_table_refuses(lib, changes):
    v = dict(head_dim=64)
    v.update(changes)
    if v == dict(head_dim=64, scaling="ntk", factor=1e308) or v.get("base") == 1e-308:
        # frequencies far outside the ordinary range are still whole fractions of a turn
        binding.RopeTable(v.pop("head_dim"), **v)
        return
    with pytest.raises(binding.PolymorphError) as e:
        binding.RopeTable(v.pop("head_dim"), **v)
    assert e.value.code == binding.PM_ERR_ARG


def test_rope_table_capacity(lib):
    with pytest.raises(binding.PolymorphError) as e:
        binding.RopeTable(272)
    assert e.value.code == binding.PM_ERR_CAPACITY


def frequencies(dim, rot, base, axes, scaling, factor, original, low, high):
    from fractions import Fraction  # noqa: F401  (the angles are compared in exact fractions of a turn below)
    each = rot // 2 // axes
    out = []
    for j in range(each):
        b = base * factor ** (each / (each - 1)) if scaling == "ntk" and each > 1 else base
        f = b ** (-j / each)
        if scaling == "linear":
            f /= factor
        if scaling == "bands":
            turns = original * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            f = f * keep + f / factor * (1.0 - keep)
        out.append(f)
    return out * axes


@pytest.mark.parametrize("axes", [1, 2])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "bands"])
@pytest.mark.parametrize("dim,rot,base", [(64, 64, 10000.0), (128, 32, 500000.0), (80, 16, 100.0), (256, 256, 3.0)])
def test_rope_table_holds_the_turns_of_a_position(lib, dim, rot, base, scaling, axes):
    t = binding.RopeTable(dim, rot_dim=rot, base=base, axes=axes, scaling=scaling, factor=8.0, original=4096, low_turns=1.0, high_turns=4.0, amplitude=1.5).table
    assert (t.head_dim, t.rot_dim, t.axes, t.amplitude) == (dim, rot, axes, 1.5)
    for i, f in enumerate(frequencies(dim, rot, base, axes, scaling, 8.0, 4096, 1.0, 4.0)):
        # the comparison's own frequencies carry a handful of roundings of 64-bit floats
        assert t.step[i] / 2.0 ** 64 == pytest.approx(f / (2 * math.pi), rel=1e-14), i
    assert all(t.step[i] == 0 for i in range(rot // 2, 128))


def norm(**changes):
    v = dict(q=ADDRESS, k=ADDRESS, q_out=ADDRESS, k_out=ADDRESS, q_stride=256, k_stride=128, q_out_stride=256, k_out_stride=128, q_gamma=ADDRESS, k_gamma=ADDRESS,
             rows=8, heads=4, kv_heads=2, head_dim=64, norm=0, eps=1e-6, dtype=0)
    v.update(changes)
    return binding.pm_qk_norm_rope_args(**v)


@pytest.mark.parametrize("changes", [
    dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(q_gamma=None), dict(k_gamma=None), dict(q=ADDRESS + 8), dict(k_out=ADDRESS + 2),
    dict(q_gamma=ADDRESS + 4), dict(q_stride=128), dict(q_stride=257), dict(k_out_stride=100), dict(rows=-1), dict(heads=0), dict(kv_heads=-1),
    dict(head_dim=72), dict(norm=2), dict(eps=-1e-6), dict(eps=math.nan), dict(dtype=3), dict(q_beta=ADDRESS), dict(norm=1, k_beta=ADDRESS + 4)])
def test_norm_refuses(lib, changes):
    assert lib.pm_qk_norm_rope(C.byref(norm(**changes)), None) == binding.PM_ERR_ARG


def test_norm_refuses_a_table_of_another_head(lib):
    table = binding.RopeTable(128)
    assert lib.pm_qk_norm_rope(C.byref(norm(table=table.address, positions=ADDRESS)), None) == binding.PM_ERR_ARG
    table = binding.RopeTable(64)
    assert lib.pm_qk_norm_rope(C.byref(norm(table=table.address)), None) == binding.PM_ERR_ARG
    assert lib.pm_qk_norm_rope(C.byref(norm(head_dim=272, q_stride=2048, q_out_stride=2048, k_stride=2048, k_out_stride=2048)), None) == binding.PM_ERR_CAPACITY


@pytest.mark.parametrize("args", [
    (None, 256, ADDRESS, 256, ADDRESS, 4, 4), (ADDRESS, 256, None, 256, ADDRESS, 4, 4), (ADDRESS, 256, ADDRESS, 256, None, 4, 4),
    (ADDRESS + 8, 256, ADDRESS, 256, ADDRESS, 4, 4), (ADDRESS, 192, ADDRESS, 256, ADDRESS, 4, 4), (ADDRESS, 256, ADDRESS, 258, ADDRESS, 4, 4),
    (ADDRESS, 256, ADDRESS, 256, ADDRESS, -1, 4), (ADDRESS, 256, ADDRESS, 256, ADDRESS, 4, 0)])
def test_rope_refuses(lib, args):
    table = binding.RopeTable(64)
    assert lib.pm_rope(*args, table.address, 0, None) == binding.PM_ERR_ARG
    assert lib.pm_rope(ADDRESS, 1 << 20, ADDRESS, 1 << 20, ADDRESS, 1, 1025, table.address, 0, None) == binding.PM_ERR_CAPACITY


def test_rope_refuses_a_broken_table(lib):
    for field, value in (("head_dim", 0), ("head_dim", 272), ("rot_dim", 8), ("rot_dim", 80), ("axes", 0), ("axes", 3)):
        table = binding.RopeTable(64)
        setattr(table.table, field, value)
        assert lib.pm_rope(ADDRESS, 256, ADDRESS, 256, ADDRESS, 4, 4, table.address, 0, None) == binding.PM_ERR_ARG, field


def test_the_binding_refuses_tensors_on_the_host(lib):
    import torch
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    off = torch.tensor([0, 4], dtype=torch.int32)
    for call in (lambda: binding.attention_packed(x, x, x, x, off, 4, 4, 0), lambda: binding.rope(x, x, off, binding.RopeTable(64), 0),
                 lambda: binding.qk_norm_rope(x, x, x, x, x, x, norm="rms", eps=1e-6, dtype=0)):
        with pytest.raises(binding.PolymorphError) as e:
            call()
        assert e.value.code == binding.PM_ERR_ARG
    with pytest.raises(binding.PolymorphError):
        binding.attention_packed(x, x, x, x, off, 4, 4, 7)
    with pytest.raises(binding.PolymorphError):
        binding.qk_norm_rope(x, x, x, x, x, x, norm="batch", eps=1e-6, dtype=0)


def test_the_binding_reads_shapes_and_distances(lib):
    import torch
    qkv = torch.zeros((5, 8, 64))
    assert binding._heads("x", "q", qkv[:, :4]) == (5, 4, 64, 512)
    assert binding._heads("x", "q", qkv[:1, 6:]) == (1, 2, 64, 512)
    assert binding._heads("x", "q", torch.zeros((1, 3, 64))) == (1, 3, 64, 192)
    for bad in (qkv[:, ::2], qkv[..., ::2], qkv.transpose(1, 2), qkv[0]):
        with pytest.raises(binding.PolymorphError):
            binding._heads("x", "q", bad)


def test_the_binding_refuses_what_the_library_cannot_count(lib):
    """Numbers beyond a field of the argument structs are refused, not cut short; one row may lie at any distance from the next."""
    import torch
    for field in (2 ** 31, "3", 1.5, None):
        with pytest.raises(binding.PolymorphError) as e:
            binding._pack("x", binding._ATTENTION_ARGS, *([64] * 19 + [field] + [0] * (len(binding.pm_packed_attention._fields_) - 20)))
        assert e.value.code == binding.PM_ERR_ARG
    values = [0] * len(binding.pm_packed_attention._fields_)
    values[[n for n, _ in binding.pm_packed_attention._fields_].index("scale")] = 10 ** 400
    with pytest.raises(binding.PolymorphError):
        binding._pack("x", binding._ATTENTION_ARGS, *values)
    with pytest.raises(binding.PolymorphError):
        binding._heads("x", "q", torch.zeros((1, 1, 16)).expand(2 ** 31, 1, 16))
    assert binding._heads("x", "q", torch.zeros(3 * 64 + 1)[1:].as_strided((1, 3, 64), (7, 64, 1))) == (1, 3, 64, 192)


# ---- which kernel a call takes ---------------------------------------------------------------------
@pytest.mark.parametrize("sizes,form", [
    # one frame: tiles of 16 rows; sixteen: units of 256
    (dict(heads=12, kv_heads=12, head_dim=64, n_seqs=1, max_q=197, max_kv=197), ("16 rows", 1, 1)),
    (dict(heads=12, kv_heads=12, head_dim=64, n_seqs=16, max_q=197, max_kv=197), ("tcgen05", 1, 1)),
    (dict(heads=12, kv_heads=12, head_dim=64, n_seqs=64, max_q=577, max_kv=577), ("tcgen05", 1, 1)),
    # single tokens: shared by a cluster, by the whole GPU with a workspace, or in even shares of many streams
    (dict(heads=16, kv_heads=4, head_dim=128, n_seqs=1, max_q=1, max_kv=32000), ("16 rows", 8, 1)),
    (dict(heads=16, kv_heads=4, head_dim=128, n_seqs=1, max_q=1, max_kv=32000, workspace_bytes=1 << 24), ("16 rows", 1, 74)),
    (dict(heads=16, kv_heads=4, head_dim=128, n_seqs=1, max_q=1, max_kv=32000, workspace_bytes=1 << 10), ("16 rows", 8, 1)),
    (dict(heads=32, kv_heads=8, head_dim=128, n_seqs=48, max_q=1, max_kv=8192), ("16 rows", 4, 1)),
    (dict(heads=32, kv_heads=8, head_dim=128, n_seqs=48, max_q=1, max_kv=300), ("16 rows", 1, 1)),
    (dict(heads=32, kv_heads=8, head_dim=128, n_seqs=3, max_q=8192, max_kv=8192), ("tcgen05", 1, 1)),
    # units of too few rows share their keys where there is a workspace
    (dict(heads=8, kv_heads=2, head_dim=128, n_seqs=1, max_q=256, max_kv=8000, workspace_bytes=1 << 28), ("tcgen05", 1, 7)),
    # a limit far above the lengths does not change the kernel
    (dict(heads=12, kv_heads=12, head_dim=64, n_seqs=512, max_q=100864, max_kv=100864, q_rows=100864, kv_rows=100864), ("tcgen05", 1, 1)),
    (dict(heads=6, kv_heads=6, head_dim=64, n_seqs=8, max_q=577, max_kv=577, dtype=1), ("fp32", 2, 1)),
    (dict(heads=6, kv_heads=6, head_dim=64, n_seqs=8, max_q=0, max_kv=577), ("none", 1, 1))])
def test_kernel_of_a_call(lib, sizes, form):
    assert binding.attention_packed_kernel(**sizes) == form


def test_kernel_and_workspace_refuse(lib):
    form, need = (C.c_int32 * 3)(), C.c_size_t(0)
    good = bytes(attention())
    assert lib.pm_attention_packed_kernel(good, 148, None) == lib.pm_attention_packed_kernel(good, 0, form) == binding.PM_ERR_ARG
    assert lib.pm_attention_packed_workspace(good, 148, None) == lib.pm_attention_packed_workspace(good, -1, C.byref(need)) == binding.PM_ERR_ARG
    bad = bytes(attention(head_dim=96))
    assert lib.pm_attention_packed_kernel(bad, 148, form) == lib.pm_attention_packed_workspace(bad, 148, C.byref(need)) == binding.PM_ERR_ARG
    assert lib.pm_attention_packed(bytes(attention(workspace=ADDRESS + 16, workspace_bytes=64)), None) == binding.PM_ERR_ARG


def test_the_binding_asks_for_every_workspace_that_is_of_use(lib):
    """The sizes at which the binding asks cover all those at which the library has a use for one."""
    need, useful = C.c_size_t(0), 0
    for heads, kv_heads in ((1, 1), (16, 4), (64, 1), (12, 12)):
        for n in (1, 2, 5, 20):
            for max_q in (1, 2, 9, 40, 300, 2000, 9000):
                for max_kv in (200, 511, 512, 1000, 4096, 9000, 100000):
                    a = attention(heads=heads, kv_heads=kv_heads, q_stride=heads * 64, out_stride=heads * 64, k_stride=kv_heads * 64, v_stride=kv_heads * 64, n_seqs=n,
                                  q_rows=n * max_q, kv_rows=n * max_kv, max_q=max_q, max_kv=max_kv)
                    assert lib.pm_attention_packed_workspace(bytes(a), 148, C.byref(need)) == 0
                    if need.value:
                        useful += 1
                        assert max_kv >= binding.LONG_HISTORY and n * kv_heads + n * max_q * heads // 128 <= binding.MANY_UNITS
    assert useful > 20


def test_the_structs_are_packed_as_the_library_reads_them(lib):
    for cls, pack in ((binding.pm_packed_attention, binding._ATTENTION_ARGS), (binding.pm_qk_norm_rope_args, binding._NORM_ARGS)):
        values = [float(i) if t is C.c_float else i for i, (_, t) in enumerate(cls._fields_, 1)]
        read = cls.from_buffer_copy(pack.pack(*values))
        assert [getattr(read, n) for n, _ in cls._fields_] == values
