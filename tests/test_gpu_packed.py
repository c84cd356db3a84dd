"""Attention over packed sequences, per-head norms with rotation, and the rotation alone, against plain statements in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {0: torch.bfloat16, 1: torch.float32}
HALF = {0: 2.0 ** -8, 1: 2.0 ** -24}          # a rounding to the type, relative


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float32)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- attention ------------------------------------------------------------------------------------------
def expected(q, k, v, causal, scale):
    """One sequence in 64 bits: the output, the mean of |v| under the same weights, and the largest sum of |q k| of a row."""
    q, k, v = q.double(), k.double(), v.double()
    group = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    n_q, n_k = len(q), len(k)
    if n_q == 0 or n_k == 0:
        return torch.zeros_like(q), torch.zeros_like(q), torch.zeros((n_q, q.shape[1], 1), dtype=torch.float64, device=q.device)
    s = torch.einsum("qhd,khd->hqk", q, k) * scale
    size = torch.einsum("qhd,khd->hqk", q.abs(), k.abs()).amax(-1) * scale
    if causal:
        hidden = torch.arange(n_k, device=q.device) > torch.arange(n_q, device=q.device)[:, None] + (n_k - n_q)
        s = s.masked_fill(hidden, -math.inf)
    p = torch.softmax(s, -1).nan_to_num(0.0)                # rows that see nothing
    return torch.einsum("hqk,khd->qhd", p, v), torch.einsum("hqk,khd->qhd", p, v.abs()), size.T[..., None]


def bound(dtype, out, mean, size, dim, n_k):
    """|error| of a row: the output's rounding; p rounded before the product (bf16); the error of a score, (dim + 4) roundings of 2^-24 of
    the sum of |q k|, enters p relatively, in numerator and denominator; sums of n_k terms in fp32 and an exponential good to 2^-22."""
    rel = 2 * (dim + 4) * 2.0 ** -24 * size + (n_k + 16) * 2.0 ** -23
    if dtype == 0:
        rel = rel + HALF[0] + 2.0 ** -16                    # products of roundings
    return HALF[dtype] * out.abs() + rel * mean + 1e-30


FILL = 7.0


def check(dtype, dim, heads, kv_heads, lengths, causal=False, *, seed=0, packed=False, gap=0, slots=False, scale=None, pad=3, size=1.0, poison=True, call=None,
          max_q=None, max_kv=None, kernel=None):
    """lengths: (queries, keys) of each sequence.  packed: q, k and v are ranges of one projection; gap: rows between sequences that belong
    to none; slots: keys in slots of a cache with kv_lengths; poison: NaN in every row that belongs to no sequence; kernel: the one that the call has
    to take."""
    from paper_2507_14959_b200 import binding
    t = TYPES[dtype]
    n_q, n_k = [a for a, _ in lengths], [b for _, b in lengths]
    q_at = np.concatenate([[0], np.cumsum(n_q)])
    rows = int(q_at[-1]) + pad
    if packed:
        assert n_q == n_k
        qkv = normal(seed, rows, heads + 2 * kv_heads, dim).mul(size).to(t).cuda()
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        k_at, kv_offsets, kv_lengths = q_at, None, None
    else:
        if slots:
            slot = max(n_k) + gap
            k_at = np.arange(len(n_k)) * slot
            kv_rows, kv_offsets, kv_lengths = slot * len(n_k), ints(k_at.tolist()), ints(n_k)
        else:
            k_at = np.concatenate([[0], np.cumsum(n_k)])
            kv_rows, kv_offsets, kv_lengths = int(k_at[-1]) + pad, ints(k_at.tolist()), None
        # a distance between rows of its own for each
        q = normal(seed, rows, heads * dim + 8).mul(size).to(t).cuda()[:, :heads * dim].unflatten(1, (heads, dim))
        k = normal(seed + 1, kv_rows, kv_heads * dim + 16).to(t).cuda()[:, :kv_heads * dim].unflatten(1, (kv_heads, dim))
        v = normal(seed + 2, kv_rows, kv_heads * dim + 24).to(t).cuda()[:, :kv_heads * dim].unflatten(1, (kv_heads, dim))
    if poison:
        q[int(q_at[-1]):] = math.nan
        live = torch.zeros(len(k), dtype=torch.bool)
        for a, b in zip(k_at, n_k):
            live[int(a):int(a) + b] = True
        k[~live.cuda()] = math.nan
        v[~live.cuda()] = math.inf
    out = torch.full((rows, heads * dim + 8), FILL, dtype=t, device="cuda")
    view = out[:, :heads * dim].unflatten(1, (heads, dim))
    status = torch.full((1,), 55, dtype=torch.int32, device="cuda")

    def run():
        binding.attention_packed(q, k, v, view, ints(q_at.tolist()), max(n_q) if max_q is None else max_q, max(n_k) if max_kv is None else max_kv, dtype, kv_offsets=kv_offsets,
                                 kv_lengths=kv_lengths, causal=causal, scale=scale, status=status)
    if kernel:
        need = 1 << 24 if kernel == "workspace" else 0
        form = binding.attention_packed_kernel(heads=heads, kv_heads=kv_heads, head_dim=dim, n_seqs=len(lengths), max_q=max(n_q) if max_q is None else max_q,
                                               max_kv=max(n_k) if max_kv is None else max_kv, q_rows=rows, kv_rows=len(k), dtype=dtype, workspace_bytes=need)
        assert form[0] == ("16 rows" if kernel in ("cluster", "workspace") else kernel), form
        assert kernel != "cluster" or form[1] > 1
        assert kernel != "workspace" or form[2] > 1
    (call or (lambda f: f()))(run)
    torch.cuda.synchronize()
    assert status.item() == 0
    assert (out[:, heads * dim:] == FILL).all() and (out[int(q_at[-1]):] == FILL).all()         # rows and columns of nobody
    for i, (a, b) in enumerate(lengths):
        at, ka = int(q_at[i]), int(k_at[i])
        want, mean, sizes = expected(q[at:at + a], k[ka:ka + b], v[ka:ka + b], causal, scale or dim ** -0.5)
        error = (view[at:at + a].double() - want).abs()
        limit = bound(dtype, want, mean, sizes, dim, b)
        assert (error <= limit).all(), (i, a, b, (error / limit).max().item())
    return view


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_short_and_odd_lengths(dtype, dim, causal):
    check(dtype, dim, 4, 2, [(n, n) for n in (1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 197)], causal, packed=True)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_empty_sequences_and_rows_that_see_nothing(dtype, dim, causal):
    check(dtype, dim, 3, 3, [(0, 0), (5, 0), (0, 7), (9, 3), (1, 1), (130, 2), (300, 40), (2, 200), (0, 0)], causal)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (12, 12, 64), (12, 4, 64), (32, 8, 128), (14, 2, 128), (8, 1, 64), (64, 1, 64), (5, 1, 128), (48, 1, 128)])
def test_grouped_heads(dtype, heads, kv_heads, dim):
    check(dtype, dim, heads, kv_heads, [(33, 33), (150, 150), (1, 1)], True, packed=True, seed=3)
    check(dtype, dim, heads, kv_heads, [(1, 300), (2, 77)], True, seed=4)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("queries", [1, 2, 5])
def test_single_tokens_over_a_cache(dtype, dim, queries):
    check(dtype, dim, 8, 2, [(queries, n) for n in (queries, 17, 500, 2049, 1000)] + [(0, 0), (queries, 4000)], True, slots=True, gap=5)


@pytest.mark.parametrize("dtype", [0, 1])
def test_one_token_of_one_stream(dtype):
    check(dtype, 128, 16, 4, [(1, 9001)], True, slots=True, gap=3)
    check(dtype, 64, 4, 4, [(1, 5)], True)
    check(dtype, 64, 3, 1, [(1, 1)], True)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 6, 6), (128, 8, 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_long_sequences(dtype, dim, heads, kv_heads, causal):
    check(dtype, dim, heads, kv_heads, [(1500, 1500), (577, 577), (700, 1900), (1900, 700)], causal, seed=9)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_growing_scores(dim, causal):
    """Peaked rows whose maximum keeps rising: what has been summed is taken down again and again."""
    check(0, dim, 4, 4, [(300, 300), (700, 700)], causal, packed=True, size=3.0, seed=21)
    check(0, dim, 4, 2, [(1, 3000), (1, 64)], causal, size=30.0, seed=22)


# Calls large enough for the tcgen05 kernel, whatever edges their sequences have.
SHORT = [(n, n) for n in (1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 197, 255, 256, 257, 320)]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_units_of_every_length(dim, causal):
    check(0, dim, 8, 8, SHORT * 12, causal, packed=True, kernel="tcgen05", seed=31)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_units_without_keys_and_rows_that_see_nothing(dim, causal):
    check(0, dim, 6, 6, [(0, 0), (5, 0), (0, 7), (9, 3), (1, 1), (130, 2), (300, 40), (2, 200), (400, 130), (256, 0), (130, 700), (0, 0)] * 14, causal, kernel="tcgen05",
          seed=32)


@pytest.mark.parametrize("heads,kv_heads,dim", [(3, 1, 64), (5, 1, 128), (14, 2, 64), (48, 1, 128), (64, 1, 64), (32, 8, 128), (33, 3, 64)])
def test_units_of_grouped_heads(heads, kv_heads, dim):
    check(0, dim, heads, kv_heads, [(1 + i * 37 % 300, 1 + i * 37 % 300 + (i % 3) * 100) for i in range(100)], True, kernel="tcgen05", seed=33)


@pytest.mark.parametrize("causal", [False, True])
def test_more_sequences_than_are_ranked(causal):
    check(0, 64, 2, 1, [(0 if i % 11 == 5 else 1 + i * 53 % 200, 1 + i * 29 % 300) for i in range(700)], causal, kernel="tcgen05", seed=34)


@pytest.mark.parametrize("dim,heads,kv_heads,count", [(64, 4, 4, 6), (128, 8, 2, 3)])
@pytest.mark.parametrize("causal", [False, True])
def test_long_units(dim, heads, kv_heads, count, causal):
    check(0, dim, heads, kv_heads, [(1500, 1500), (577, 577), (700, 1900), (1900, 700), (2111, 2111)] * count, causal, kernel="tcgen05", seed=35)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_units_with_growing_scores(dim, causal):
    """Rows whose maximum keeps rising by more than the lag that the kernel allows: their sums and outputs are taken down."""
    from paper_2507_14959_b200 import binding
    n, heads = 1024, 10
    assert binding.attention_packed_kernel(heads=heads, kv_heads=heads, head_dim=dim, n_seqs=2, max_q=n, max_kv=n)[0] == "tcgen05"
    q, k, v = (normal(40 + i, 2 * n, heads, dim) for i in range(3))
    k = k * (1 + torch.arange(2 * n).view(-1, 1, 1) % n / 60.0)                # keys grow along the sequence: 1 to 18 times
    q[5::7] *= 4
    q, k, v = (x.bfloat16().cuda() for x in (q, k, v))
    out, status = torch.zeros_like(q), ints([0])
    binding.attention_packed(q, k, v, out, ints([0, n, 2 * n]), n, n, 0, causal=causal, status=status)
    assert status.item() == 0
    for a in (0, n):
        want, mean, size = expected(q[a:a + n], k[a:a + n], v[a:a + n], causal, dim ** -0.5)
        error, limit = (out[a:a + n].double() - want).abs(), bound(0, want, mean, size, dim, n)
        assert (error <= limit).all(), (error / limit).max()


def test_values_that_are_not_numbers_stay_in_their_rows():
    """A NaN in a query is in its row's output alone, one in a key in the outputs of the rows that see it; hidden keys may hold anything."""
    from paper_2507_14959_b200 import binding
    for n, seqs, kernel in ((40, 1, "16 rows"), (300, 12, "tcgen05")):
        heads, dim = 4, 64
        assert binding.attention_packed_kernel(heads=heads, kv_heads=heads, head_dim=dim, n_seqs=seqs, max_q=n, max_kv=n)[0] == kernel
        q, k, v = (normal(50 + i, seqs * n, heads, dim).bfloat16().cuda() for i in range(3))
        off, out = ints([i * n for i in range(seqs + 1)]), torch.zeros_like(q)
        binding.attention_packed(q, k, v, out, off, n, n, 0, causal=True)
        plain = out.clone()
        q[7, 1] = math.nan
        k[n - 3, 2] = math.nan
        binding.attention_packed(q, k, v, out, off, n, n, 0, causal=True)
        bad = torch.zeros_like(out, dtype=torch.bool)
        bad[7, 1] = True
        bad[n - 3:n, 2] = True
        assert torch.isnan(out[bad]).all() and torch.equal(out[~bad], plain[~bad])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("queries", [1, 3])
def test_a_long_history_shared_through_a_workspace(dim, queries):
    check(0, dim, 16, 4, [(queries, 20001)], True, slots=True, gap=7, kernel="workspace", seed=61)
    check(0, dim, 4, 2, [(queries, 9000), (0, 0), (queries, 17), (queries, 0)], True, slots=True, gap=7, kernel="workspace", seed=62)
    check(0, dim, 4, 2, [(queries, 5001), (queries, 4444)], False, kernel="workspace", seed=63)


def test_a_workspace_that_is_too_small_or_missing():
    """The library itself: with less than it asks for it takes clusters, with enough the workspace; nothing behind it is written."""
    import ctypes as C
    from paper_2507_14959_b200 import binding
    lib, heads, kv_heads, dim, n = binding.load(), 8, 2, 64, 12000
    q, k, v = normal(1, 1, heads, dim).bfloat16().cuda(), normal(2, n, kv_heads, dim).bfloat16().cuda(), normal(3, n, kv_heads, dim).bfloat16().cuda()
    q_off, k_off = ints([0, 1]), ints([0, n])
    want, mean, size = expected(q, k, v, True, dim ** -0.5)
    limit = bound(0, want, mean, size, dim, n)

    def args(space, count):
        out = torch.full_like(q, FILL)
        return out, binding._ATTENTION_ARGS.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), heads * dim, kv_heads * dim, kv_heads * dim, heads * dim,
                                                 q_off.data_ptr(), k_off.data_ptr(), 0, 1, n, 1, 1, n, heads, kv_heads, dim, 1, 0.0, 0, 0, space, count)
    need = C.c_size_t(0)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert lib.pm_attention_packed_workspace(args(0, 0)[1], sms, C.byref(need)) == 0 and need.value > 0
    for have in (0, 16, need.value - 16, need.value):
        space = torch.full((need.value + 4096,), 77, dtype=torch.uint8, device="cuda")
        out, packed = args(space.data_ptr() if have else 0, have)
        assert lib.pm_attention_packed(packed, binding._stream_ptr(None)) == 0
        torch.cuda.synchronize()
        assert ((out.double() - want).abs() <= limit).all(), have
        assert (space[need.value:] == 77).all() and ((space[:need.value] == 77).all().item() == (have < need.value))


def test_graphs_replayed_side_by_side_share_no_workspace():
    from paper_2507_14959_b200 import binding
    n, heads, kv_heads, dim = 15000, 8, 2, 128
    streams, graphs, calls = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for i, s in enumerate(streams):
        q, k, v = normal(i, 1, heads, dim).bfloat16().cuda(), normal(10 + i, n, kv_heads, dim).bfloat16().cuda(), normal(20 + i, n, kv_heads, dim).bfloat16().cuda()
        out, q_off, k_off = torch.zeros_like(q), ints([0, 1]), ints([0, n])
        call = lambda q=q, k=k, v=v, out=out, q_off=q_off, k_off=k_off: binding.attention_packed(q, k, v, out, q_off, 1, n, 0, kv_offsets=k_off, causal=True)  # noqa: E731
        with torch.cuda.stream(s):
            call()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                call()
        graphs.append((g, call))                       # the call's buffers, its lists among them, outlive the replays
        calls.append((q, k, v, out))
    for turn in range(20):
        for q, k, v, out in calls:
            q.copy_(normal(100 + turn, *q.shape))
            out.zero_()
        torch.cuda.synchronize()
        for s, (g, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        if turn % 5 == 0:
            for q, k, v, out in calls:
                want, mean, size = expected(q, k, v, True, dim ** -0.5)
                assert ((out.double() - want).abs() <= bound(0, want, mean, size, dim, n)).all()


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_scale_of_its_own(dtype):
    check(dtype, 64, 2, 2, [(100, 100), (1, 1)], True, packed=True, scale=0.5)
    check(dtype, 128, 2, 2, [(1, 100)], True, scale=0.01)


def test_many_short_sequences():
    check(0, 64, 3, 3, [(1 + i * 7 % 40, 1 + i * 7 % 40) for i in range(600)], False, packed=True, seed=5)


def test_ragged_frames():
    check(0, 64, 12, 12, [(65 + i * 157 % 513, 65 + i * 157 % 513) for i in range(40)], False, packed=True, seed=6)


def test_bounds_larger_than_the_lists_need():
    check(0, 64, 4, 4, [(40, 40), (3, 3)], True, packed=True, max_q=4000, max_kv=100000)
    check(0, 128, 4, 1, [(2, 90)], True, max_q=43, max_kv=93)
    check(1, 64, 4, 4, [(40, 40), (3, 3)], True, packed=True, max_q=4000, max_kv=100000)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("queries", [1, 40, 300])
def test_malformed_lists_are_skipped(dtype, queries):
    """A sequence whose list is wrong is left out, its rows of the output as they were; the others are served."""
    from paper_2507_14959_b200 import binding
    t, n = TYPES[dtype], queries
    q, k, v = (normal(i, 4 * n, 2, 64).to(t).cuda() for i in range(3))
    good = [0, n, 2 * n, 3 * n, 4 * n]

    def run(q_offsets, kv_offsets, kv_lengths, max_q=n, max_kv=4 * n):
        out = torch.full_like(q, FILL)
        status = ints([0])
        binding.attention_packed(q, k, v, out, ints(q_offsets), max_q, max_kv, dtype, kv_offsets=None if kv_offsets is None else ints(kv_offsets),
                                 kv_lengths=None if kv_lengths is None else ints(kv_lengths), causal=True, status=status)
        torch.cuda.synchronize()
        return out, status.item()

    whole, status = run(good, good, None)
    assert status == 0
    for kv_offsets, kv_lengths in (([0, n, 2 * n, -1], [n] * 4), ([0, n, 2 * n, 3 * n], [n, n, n, n + 1]), ([0, n, 2 * n, 3 * n], [n, n, n, -1]),
                                   ([0, n, 2 * n, 2 ** 31 - 1], [n] * 4), ([0, n, 2 * n, 4 * n + 1], [n] * 3 + [0]), (good[:3] + [3 * n, 3 * n - 1], None)):
        out, status = run(good, kv_offsets, kv_lengths)
        assert status == binding.PM_ERR_ARG
        assert (out[3 * n:] == FILL).all() and torch.equal(out[:3 * n], whole[:3 * n]), kv_offsets
    for q_offsets in ([0, n, 2 * n, 3 * n, 4 * n + 1], [0, n, 2 * n, 3 * n, -5], [0, n, 2 * n, 3 * n, 2 ** 31 - 1], [0, n, 2 * n, 3 * n, 2 * n]):
        out, status = run(q_offsets, [0, n, 2 * n, 3 * n], [n] * 4)
        assert status == binding.PM_ERR_ARG
        assert (out[3 * n:] == FILL).all() and torch.equal(out[:3 * n], whole[:3 * n]), q_offsets
    # longer than the call's limits.  Fewer sequences or another limit may split the keys otherwise: every call's rows lie within the bound of the
    # exact ones, not on one another's bits
    def served(out, sequences):
        for i in range(sequences):
            at = slice(i * n, (i + 1) * n)
            want, mean, sizes = expected(q[at], k[at], v[at], True, 0.125)
            assert ((out[at].double() - want).abs() <= bound(dtype, want, mean, sizes, 64, n)).all()
    served(whole, 4)
    out, status = run([0, n, 2 * n, 4 * n], good[:3], [n, n, n])
    assert status == binding.PM_ERR_ARG and (out[2 * n:] == FILL).all()
    served(out, 2)
    out, status = run(good, good[:4], [n, n, n, 4 * n], max_kv=4 * n - 1)
    assert status == binding.PM_ERR_ARG and (out[3 * n:] == FILL).all()
    served(out, 3)


@pytest.mark.parametrize("lengths", [[(1, 700)], [(200, 200), (90, 90)]])
def test_a_captured_call_replays_with_other_lengths_and_values(lengths):
    from paper_2507_14959_b200 import binding
    n_q, n_k = sum(a for a, _ in lengths), sum(b for _, b in lengths)
    q, k, v = normal(1, n_q, 4, 64).bfloat16().cuda(), normal(2, n_k, 2, 64).bfloat16().cuda(), normal(3, n_k, 2, 64).bfloat16().cuda()
    q_off = ints(np.concatenate([[0], np.cumsum([a for a, _ in lengths])]).tolist())
    k_off = ints(np.concatenate([[0], np.cumsum([b for _, b in lengths])]).tolist())
    k_len = ints([b for _, b in lengths])
    out, status = torch.zeros_like(q), ints([0])

    def call():
        binding.attention_packed(q, k, v, out, q_off, max(a for a, _ in lengths), max(b for _, b in lengths), 0, kv_offsets=k_off, kv_lengths=k_len, causal=True,
                                 status=status)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
    for turn in range(3):
        if turn:
            q.copy_(normal(10 + turn, *q.shape))
            k_len.copy_(ints([b - 13 * turn for _, b in lengths]))
        out.fill_(FILL)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, replayed) and status.item() == 0
        for i, (a, b) in enumerate(lengths):
            b -= 13 * turn
            at, ka = int(q_off[i]), int(k_off[i])
            want, mean, sizes = expected(q[at:at + a], k[ka:ka + b], v[ka:ka + b], True, 0.125)
            assert ((replayed[at:at + a].double() - want).abs() <= bound(0, want, mean, sizes, 64, b)).all()


def test_first_calls_of_a_process_may_be_captured():
    """Nothing is set up by a first call that a capture could not hold."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2507_14959_b200 import binding
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
x = torch.randn(600, 8, 64, device="cuda").bfloat16()
table, at, g1 = binding.RopeTable(64), ints(list(range(600))), torch.ones(64, device="cuda")
outs = [torch.zeros_like(x) for _ in range(5)]
few, all_, hist = ints([0, 3]), ints([0, 100, 600]), ints([0, 600])
def calls(o):
    binding.rope(x, o[0], at, table, 0)
    binding.qk_norm_rope(x, None, o[1], None, g1, None, norm="rms", eps=1e-6, dtype=0, positions=at, table=table)
    binding.attention_packed(x, x, x, o[2], few, 3, 600, 0, kv_offsets=hist, causal=True)
    binding.attention_packed(x, x, x, o[3], all_, 500, 500, 0)
    f = x.float()
    binding.attention_packed(f, f, f, o[4].float(), all_, 500, 500, 1)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls(outs)
graph.replay()
torch.cuda.synchronize()
eager = [torch.zeros_like(x) for _ in range(5)]
calls(eager)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(outs, eager)) and outs[3].abs().sum() > 0
print("captured")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "captured" in done.stdout, done.stderr[-2000:]


def test_a_workspace_on_another_stream_than_torchs():
    """The call's stream is given, torch's current one is busy with memory it has already given back: the workspace is none of that."""
    from paper_2507_14959_b200 import binding
    n, heads, kv_heads, dim = 16000, 8, 2, 128
    q, k, v = normal(1, 1, heads, dim).bfloat16().cuda(), normal(2, n, kv_heads, dim).bfloat16().cuda(), normal(3, n, kv_heads, dim).bfloat16().cuda()
    out, q_off, k_off, other = torch.zeros_like(q), ints([0, 1]), ints([0, n]), torch.cuda.Stream()
    want, mean, size = expected(q, k, v, True, dim ** -0.5)
    kept = torch.zeros(1 << 20, device="cuda")
    torch.cuda.synchronize()
    for turn in range(5):
        torch.cuda._sleep(20_000_000)                      # the current stream is behind
        lent = torch.full((1 << 20,), float(turn + 1), device="cuda")
        kept.copy_(lent)
        del lent                                           # its memory may be given out again on the current stream
        binding.attention_packed(q, k, v, out, q_off, 1, n, 0, kv_offsets=k_off, causal=True, stream=other if turn % 2 else other.cuda_stream)
        torch.cuda.synchronize()
        assert (kept == turn + 1).all()
        assert ((out.double() - want).abs() <= bound(0, want, mean, size, dim, n)).all()


def test_units_that_share_their_keys():
    """Few units over long histories: their keys are cut into parts, which a second kernel joins."""
    from paper_2507_14959_b200 import binding
    for dim, heads, kv_heads, lengths in ((128, 8, 2, [(256, 8000)]), (64, 4, 4, [(3000, 8192), (0, 500), (257, 0), (5, 5000)]), (64, 6, 2, [(700, 9000), (90, 300)]),
                                          (128, 5, 5, [(4096, 4096)])):
        for causal in (True, False):
            form = binding.attention_packed_kernel(heads=heads, kv_heads=kv_heads, head_dim=dim, n_seqs=len(lengths), max_q=max(a for a, _ in lengths),
                                                   max_kv=max(b for _, b in lengths), q_rows=sum(a for a, _ in lengths) + 3, kv_rows=sum(b for _, b in lengths) + 3,
                                                   workspace_bytes=1 << 28)
            if causal:
                assert form[0] == "tcgen05" and form[2] > 1, form
            check(0, dim, heads, kv_heads, lengths, causal, seed=71)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("queries,form", [(700, "tcgen05"), (2, "16 rows")])
def test_parts_in_a_workspace_that_held_something_else(queries, form, causal):
    """The library itself, with a workspace full of NaN: sequences without keys and rows that see nothing give zeros, a malformed sequence's rows stay, a
    NaN stays in its row, nothing behind the workspace is written."""
    import ctypes as C
    from paper_2507_14959_b200 import binding
    heads, kv_heads, dim, n = 4, 2, 64, 9000
    lengths, long_last = [(queries, n), (queries, 0), (queries, queries // 2), (queries, 70)], (queries, 5000)
    q_at = np.cumsum([0] + [a for a, _ in lengths] + [queries])
    k_at = np.cumsum([0] + [b for _, b in lengths])
    rows, kv_rows = int(q_at[-1]), int(k_at[-1])
    q, k, v = normal(1, rows, heads, dim).bfloat16().cuda(), normal(2, kv_rows, kv_heads, dim).bfloat16().cuda(), normal(3, kv_rows, kv_heads, dim).bfloat16().cuda()
    q[1, 2] = math.nan
    # the last sequence's keys would lie behind the buffer
    q_off, k_off, counts = ints(q_at.tolist()), ints(k_at.tolist()), ints([b for _, b in lengths] + [long_last[1]])
    out, status = torch.full_like(q, FILL), ints([0])
    lib, sms, need = binding.load(), torch.cuda.get_device_properties(0).multi_processor_count, C.c_size_t(0)
    fields = (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), heads * dim, kv_heads * dim, kv_heads * dim, heads * dim, q_off.data_ptr(), k_off.data_ptr(),
              counts.data_ptr(), rows, kv_rows, len(lengths) + 1, queries, n, heads, kv_heads, dim, int(causal), 0.0, 0, status.data_ptr())
    assert lib.pm_attention_packed_workspace(binding._ATTENTION_ARGS.pack(*fields, 0, 0), sms, C.byref(need)) == 0 and need.value > 0
    space = torch.full((need.value + 4096,), 255, dtype=torch.uint8, device="cuda")         # every float a NaN
    packed, took = binding._ATTENTION_ARGS.pack(*fields, space.data_ptr(), need.value), (C.c_int32 * 3)()
    assert lib.pm_attention_packed_kernel(packed, sms, took) == 0 and (took[0], took[2] > 1) == (("16 rows", "tcgen05").index(form), True)
    assert lib.pm_attention_packed(packed, binding._stream_ptr(None)) == 0
    torch.cuda.synchronize()
    assert status.item() == binding.PM_ERR_ARG and (out[rows - queries:] == FILL).all() and (space[need.value:] == 255).all()
    assert torch.isnan(out[1, 2]).all()
    out[1, 2] = q[1, 2] = 0
    for (a, b), x, y in zip(lengths, q_at, k_at):
        want, mean, size = expected(q[x:x + a], k[y:y + b], v[y:y + b], causal, dim ** -0.5)
        if x == 0:
            want[1, 2] = 0
        assert ((out[x:x + a].double() - want).abs() <= bound(0, want, mean, size, dim, max(b, 1))).all(), (a, b)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("causal", [True, False])
def test_limits_far_above_the_lengths(dtype, causal):
    """max_q = all rows: a sequence's tiles are more than the grid gives it, and most sequences leave most of theirs empty."""
    from paper_2507_14959_b200 import binding
    lengths = [(3, 3)] * 1500 + [(500, 500)] + [(17, 17), (0, 0), (1, 1)] * 30
    rows = sum(a for a, _ in lengths)
    form = binding.attention_packed_kernel(heads=4, kv_heads=2, head_dim=64, n_seqs=len(lengths), max_q=rows, max_kv=rows, q_rows=rows, kv_rows=rows, dtype=dtype)
    assert form[0] == ("fp32" if dtype else "16 rows") and form[2] == 1, form
    q_off = [0]
    for n, _ in lengths:
        q_off.append(q_off[-1] + n)
    q, k, v = (normal(s, rows, h, 64).to(torch.float32 if dtype else torch.bfloat16).cuda() for s, h in ((1, 4), (2, 2), (3, 2)))
    tight, loose, status = torch.full_like(q, 7), torch.full_like(q, 7), ints([5])
    binding.attention_packed(q, k, v, tight, ints(q_off), 500, 500, dtype, causal=causal)
    binding.attention_packed(q, k, v, loose, ints(q_off), rows, rows, dtype, causal=causal, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    for n, at in zip((n for n, _ in lengths), q_off):
        if n == 0:
            continue
        want, mean, size = expected(q[at:at + n], k[at:at + n], v[at:at + n], causal, 64 ** -0.5)
        for out in (tight, loose):
            assert ((out[at:at + n].double() - want).abs() <= bound(dtype, want, mean, size, 64, n)).all()


def test_other_streams_side_by_side():
    """Calls on two streams share nothing."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    views = []
    for turn in range(6):
        def on(f, s=streams[turn % 2]):
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                f()
        views.append(check(0, 64, 4, 2, [(200, 200), (1, 900)] if turn < 3 else [(1, 900)], True, seed=turn // 2, call=on))
    from paper_2507_14959_b200 import binding
    q, k, v = (normal(i, 500, 4, 64).bfloat16().cuda() for i in range(3))
    alone = torch.zeros_like(q)
    off = ints([0, 300, 301, 500])
    binding.attention_packed(q, k, v, alone, off, 300, 300, 0)
    outs = [torch.zeros_like(q) for _ in range(8)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        binding.attention_packed(q, k, v, o, off, 300, 300, 0, stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(alone, o) for o in outs)


def test_results_do_not_depend_on_the_run():
    a = check(0, 128, 8, 2, [(1, 5000), (3, 77)], True, seed=2).clone()
    b = check(0, 128, 8, 2, [(1, 5000), (3, 77)], True, seed=2)
    assert torch.equal(a, b)


def test_rows_beyond_the_32_bit_range():
    """Keys whose distance from the cache's start passes 2^31 elements."""
    from paper_2507_14959_b200 import binding
    dim, kv_heads, rows = 128, 8, 2_300_000                 # 2.36e9 elements, 4.7 GB
    cache = torch.zeros((rows, kv_heads, dim), dtype=torch.bfloat16, device="cuda")
    start, n = rows - 700, 700
    k, v = normal(1, n, kv_heads, dim).bfloat16().cuda(), normal(2, n, kv_heads, dim).bfloat16().cuda()
    for queries in (1, 300):
        q = normal(3, queries, 16, dim).bfloat16().cuda()
        outs = []
        for source in (k, v):
            cache[start:] = source
            out = torch.zeros_like(q)
            binding.attention_packed(q, cache, cache, out, ints([0, queries]), queries, n, 0, kv_offsets=ints([start]), kv_lengths=ints([n]), causal=True)
            want = torch.zeros_like(q)
            binding.attention_packed(q, source, source, want, ints([0, queries]), queries, n, 0, kv_offsets=ints([0]), kv_lengths=ints([n]), causal=True)
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            outs.append(out)
        assert not torch.equal(*outs)


def test_nothing_to_do():
    from paper_2507_14959_b200 import binding
    x = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    status = ints([9])
    binding.attention_packed(x, x, x, x, ints([0]), 0, 0, 0, status=status)
    assert status.item() == 0
    q = torch.full((3, 2, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, FILL)
    binding.attention_packed(q, x, x, out, ints([0, 2]), 2, 0, 0, kv_offsets=ints([0, 0]), status=status)
    torch.cuda.synchronize()
    assert status.item() == 0 and (out[:2] == 0).all() and (out[2:] == FILL).all()


def test_a_stream_of_nobody_is_refused_by_type():
    from paper_2507_14959_b200 import binding
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    off = ints([0, 4])
    for bad in (lambda: binding.attention_packed(q.float(), q, q, q, off, 4, 4, 0), lambda: binding.attention_packed(q, q, q, q, off.long(), 4, 4, 0),
                lambda: binding.attention_packed(q, q, q[:3], q, off, 4, 4, 0), lambda: binding.attention_packed(q, q, q, q.transpose(1, 2), off, 4, 4, 0),
                lambda: binding.attention_packed(q, q, q, q, off, 4, 4, 0, kv_lengths=ints([1])),
                lambda: binding.attention_packed(q, q, q, q, off, 4, 4, 0, kv_offsets=ints([0]), kv_lengths=ints([1, 2]))):
        with pytest.raises(binding.PolymorphError) as e:
            bad()
        assert e.value.code == binding.PM_ERR_ARG


# ---- rotation, with and without norms ---------------------------------------------------------------------
def frequencies(rot, base, axes, scaling, factor, original, low, high):
    each = rot // 2 // axes
    j = torch.arange(each, dtype=torch.float64)
    if scaling == "ntk" and each > 1:
        base = base * factor ** (each / (each - 1))
    f = torch.exp(-j / each * math.log(base))
    if scaling == "linear":
        f = f / factor
    if scaling == "bands":
        turns = original * f / (2 * math.pi)
        keep = ((turns - low) / (high - low)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    return f.cuda()


def rotated(x, positions, rot, interleaved, axes, f, amplitude):
    """x in 64 bits; also |a| + |b| of each element's pair."""
    angle = (positions.double().view(-1, axes, 1) * f).flatten(1)[:, None]
    c, s = amplitude * angle.cos(), amplitude * angle.sin()
    y, size = x.clone(), x.abs()
    at = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    size = size.clone()
    size[..., at[0]] = size[..., at[1]] = (a.abs() + b.abs()) * abs(amplitude)
    return y, size


ROPE_CASES = [
    # dim, rot, interleaved, axes, scaling, far
    (64, 64, False, 1, "none", 1000), (64, 64, True, 2, "none", 40), (128, 64, True, 1, "linear", 100000), (128, 128, False, 2, "bands", 100),
    (80, 80, False, 1, "ntk", 5000), (80, 32, True, 2, "bands", 3000), (96, 16, False, 1, "none", 10), (16, 16, True, 1, "none", 50), (32, 32, False, 2, "none", 14),
    (256, 256, True, 1, "bands", 2 ** 31 - 1), (48, 32, False, 2, "ntk", 100), (256, 16, False, 1, "none", 2 ** 30)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dim,rot,interleaved,axes,scaling,far", ROPE_CASES)
@pytest.mark.parametrize("rows,heads", [(1, 1), (37, 5), (600, 12)])
def test_rope(dtype, dim, rot, interleaved, axes, scaling, far, rows, heads):
    from paper_2507_14959_b200 import binding
    t = TYPES[dtype]
    table = binding.RopeTable(dim, rot_dim=rot, base=500.0, interleaved=interleaved, axes=axes, scaling=scaling, factor=4.0, original=2000, low_turns=1.0,
                              high_turns=3.0, amplitude=1.25)
    wide = normal(rows, rows + 2, heads * dim + 24).to(t).cuda()
    x = wide[:rows, :heads * dim].unflatten(1, (heads, dim))
    g = torch.Generator().manual_seed(rows)
    positions = torch.randint(-far, far, (rows, axes) if axes == 2 else (rows,), generator=g).int()
    positions.view(-1)[0] = far
    positions = positions.cuda()
    out = torch.full((rows + 2, heads * dim + 8), FILL, dtype=t, device="cuda")
    y = out[:rows, :heads * dim].unflatten(1, (heads, dim))
    binding.rope(x, y, positions, table, dtype)
    torch.cuda.synchronize()
    want, size = rotated(x.double(), positions, rot, interleaved, axes, frequencies(rot, 500.0, axes, scaling, 4.0, 2000, 1.0, 3.0), 1.25)
    # sine and cosine to 2 units of 2^-24 and the angle's last bit, two products and their sum; the comparison's own angles in 64 bits are off
    # by 2^-52 of theirs; behind the rotated part nothing changes
    limit = HALF[dtype] * want.abs() + (2.0 ** -21 + abs(far) * 2.0 ** -50) * size
    limit[..., rot:] = 0
    assert ((y.double() - want).abs() <= limit).all()
    assert (out[rows:] == FILL).all() and (out[:, heads * dim:] == FILL).all()
    again = x.clone()
    binding.rope(again, again, positions, table, dtype)                       # in place
    assert torch.equal(again, y)
    binding.rope(x, x, positions, table, dtype)                               # in place within the wide buffer
    assert torch.equal(x, y)


def normed(x, gamma, beta, kind, eps):
    """The norm in 64 bits; also the size that its roundings are relative to."""
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    inv = torch.rsqrt((x - mean).square().mean(-1, keepdim=True) + eps)
    u = (x - mean) * inv * gamma
    size = x.abs().amax(-1, keepdim=True) * inv * gamma.abs()
    if beta is not None:
        u, size = u + beta, size + beta.abs()
    return u, size


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("kind,with_beta,per_head", [("rms", False, False), ("rms", False, True), ("layer", True, False), ("layer", False, True), ("layer", True, True)])
@pytest.mark.parametrize("dim,rot,interleaved,axes", [(64, 64, False, 2), (128, 64, True, 1), (80, 80, False, 1), (256, 128, True, 2), (64, 0, False, 1)])
@pytest.mark.parametrize("rows,heads,kv_heads", [(1, 3, 3), (45, 12, 4), (700, 6, 0)])
def test_norm_with_rotation(dtype, kind, with_beta, per_head, dim, rot, interleaved, axes, rows, heads, kv_heads):
    from paper_2507_14959_b200 import binding
    t = TYPES[dtype]
    table = binding.RopeTable(dim, rot_dim=rot, base=100.0, interleaved=interleaved, axes=axes, amplitude=1.1) if rot else None
    positions = torch.randint(0, 5000, (rows, axes) if axes == 2 else (rows,), generator=torch.Generator().manual_seed(1)).int().cuda() if rot else None
    qkv = (normal(rows, rows, heads + 2 * kv_heads, dim) * 2 + 0.5).to(t).cuda()
    q, k = qkv[:, :heads], qkv[:, heads:heads + kv_heads] if kv_heads else None
    gamma = {n: 1 + 0.3 * normal(i, *((h, dim) if per_head else (dim,))).cuda() for i, (n, h) in enumerate((("q", heads), ("k", kv_heads)))}
    beta = {n: 0.3 * normal(5 + i, *((h, dim) if per_head else (dim,))).cuda() if with_beta else None for i, (n, h) in enumerate((("q", heads), ("k", kv_heads)))}
    q_out = torch.full((rows, heads, dim), FILL, dtype=t, device="cuda")
    k_out = torch.full((rows, kv_heads, dim), FILL, dtype=t, device="cuda") if kv_heads else None
    values = qkv[:, heads + kv_heads:].clone()

    def call(q, k, qo, ko):
        binding.qk_norm_rope(q, k, qo, ko, gamma["q"], gamma["k"] if kv_heads else None, norm=kind, eps=1e-5, dtype=dtype, q_beta=beta["q"],
                             k_beta=beta["k"] if kv_heads else None, positions=positions, table=table)
    call(q, k, q_out, k_out)
    torch.cuda.synchronize()
    for name, x, y in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            continue
        u, size = normed(x.double(), gamma[name].double(), None if beta[name] is None else beta[name].double(), kind, 1e-5)
        if rot:
            f = frequencies(rot, 100.0, axes, "none", 1.0, 0, 0, 1)
            want, _ = rotated(u, positions, rot, interleaved, axes, f, 1.1)
            size = 2.2 * size.amax(-1, keepdim=True)
        else:
            want = u
        # sums of dim terms in fp32 (each rounding relative to the head's largest element), then as the rotation's
        limit = HALF[dtype] * want.abs() + ((dim + 16) * 2.0 ** -23 + 2.0 ** -21) * size
        assert ((y.double() - want).abs() <= limit).all(), name
    call(q, k, q, k)                                                          # in place: the values behind stay as they were
    torch.cuda.synchronize()
    assert torch.equal(q, q_out) and (k is None or torch.equal(k, k_out)) and torch.equal(qkv[:, heads + kv_heads:], values)


def test_rope_captured():
    from paper_2507_14959_b200 import binding
    table = binding.RopeTable(64)
    x, positions = normal(1, 30, 4, 64).bfloat16().cuda(), ints(list(range(30)))
    y = torch.zeros_like(x)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        binding.rope(x, y, positions, table, 0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            binding.rope(x, y, positions, table, 0)
    del table
    positions += 5
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    want = torch.zeros_like(x)
    binding.rope(x, want, positions, binding.RopeTable(64), 0)
    assert torch.equal(y, want)


# ---- together ---------------------------------------------------------------------------------------------
def test_a_block_of_an_encoder_over_frames_of_different_sizes():
    """qkv projection -> norms with rotation by row and column -> attention over the packed frames -> output projection with the residual, as one
    block runs them, all in place in one qkv buffer; against the same steps in 64 bits with the stored roundings between them."""
    from paper_2507_14959_b200 import binding
    heads, dim, grids = 6, 64, [(14, 14), (7, 9), (1, 1), (24, 24), (3, 50)]
    d, tokens = heads * dim, [a * b for a, b in grids]
    rows, off = sum(tokens), np.concatenate([[0], np.cumsum(tokens)]).tolist()
    positions = ints([[i // b, i % b] for a, b in grids for i in range(a * b)])
    x = normal(1, rows, d).bfloat16().cuda()
    w_qkv, w_out = normal(2, d, 3 * d).mul(0.05).bfloat16().float().numpy(), normal(3, d, d).mul(0.05).bfloat16().float().numpy()
    bias = np.zeros(3 * d, np.float32)
    none, no_ids = np.zeros(2, np.int32), np.zeros(0, np.int32)
    lin_qkv = binding.Linear(w_qkv, bias, max_adapters=1, max_rank=16, max_set=1, max_frames=1, tokens=rows)
    lin_out = binding.Linear(w_out, bias[:d], max_adapters=1, max_rank=16, max_set=1, max_frames=1, tokens=rows, epilogue=2)
    table = binding.RopeTable(dim, base=100.0, axes=2)
    gamma = 1 + 0.2 * normal(4, 2, dim).cuda()
    qkv = torch.zeros((rows, 3 * heads, dim), dtype=torch.bfloat16, device="cuda")
    mixed, y = torch.zeros((rows, heads, dim), dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x)
    lin_qkv.forward(x, 1, none, no_ids, qkv)
    made = qkv.clone()
    q, k, v = qkv[:, :heads], qkv[:, heads:2 * heads], qkv[:, 2 * heads:]
    binding.qk_norm_rope(q, k, q, k, gamma[0], gamma[1], norm="rms", eps=1e-6, dtype=0, positions=positions, table=table)
    binding.attention_packed(q, k, v, mixed, ints(off), max(tokens), max(tokens), 0)
    lin_out.forward(mixed, 1, none, no_ids, y, residual=x)
    torch.cuda.synchronize()
    assert lin_out.status() == 0
    f = frequencies(dim, 100.0, 2, "none", 1.0, 0, 0, 1)
    for i, name in enumerate(("q", "k")):
        u, size = normed(made[:, i * heads:(i + 1) * heads].double(), gamma[i].double(), None, "rms", 1e-6)
        want, _ = rotated(u, positions, dim, False, 2, f, 1.0)
        got = (q, k)[i]
        assert ((got.double() - want).abs() <= HALF[0] * want.abs() + 80 * 2.0 ** -22 * size.amax(-1, keepdim=True)).all(), name
    assert torch.equal(v, made[:, 2 * heads:])
    for a, b in zip(off, off[1:]):
        want, mean, sizes = expected(q[a:b], k[a:b], v[a:b], False, dim ** -0.5)
        assert ((mixed[a:b].double() - want).abs() <= bound(0, want, mean, sizes, dim, b - a)).all()
    m = mixed.double().flatten(1)
    want = m @ torch.from_numpy(w_out).double().cuda() + x.double()
    size = m.abs() @ torch.from_numpy(w_out).double().abs().cuda() + x.double().abs()
    assert ((y.double() - want).abs() <= HALF[0] * want.abs() + (d + 4) * 2.0 ** -23 * size).all()


def test_a_stream_that_keeps_its_tokens():
    """Token by token and in chunks over a cache: the same rows as the whole clip at once, to the operator's own error."""
    from paper_2507_14959_b200 import binding
    heads, kv_heads, dim, n = 8, 2, 128, 150
    q, k, v = normal(1, n, heads, dim).bfloat16().cuda(), normal(2, n, kv_heads, dim).bfloat16().cuda(), normal(3, n, kv_heads, dim).bfloat16().cuda()
    cache = torch.full((2, 200, kv_heads, dim), math.nan, dtype=torch.bfloat16, device="cuda")
    got = torch.zeros_like(q)
    at = 0
    for step in (1, 1, 70, 1, 17, 60):
        cache[0, at:at + step], cache[1, at:at + step] = k[at:at + step], v[at:at + step]
        binding.attention_packed(q[at:at + step], cache[0], cache[1], got[at:at + step], ints([0, step]), step, 200, 0, kv_offsets=ints([0]),
                                 kv_lengths=ints([at + step]), causal=True)
        at += step
    assert at == n
    want, mean, sizes = expected(q, k, v, True, dim ** -0.5)
    assert ((got.double() - want).abs() <= bound(0, want, mean, sizes, dim, n)).all()
