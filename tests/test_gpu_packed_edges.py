"""Edges of the packed-sequence operators: what goes before a call, what it reports, forms that the larger tests do not reach."""
import numpy as np
import pytest
import torch

from test_gpu_packed import bound, check, expected, ints, normal

pytestmark = pytest.mark.gpu


def fail_a_call():
    """A library call that fails on the host: adapter tables of 512 GB, refused by the allocator."""
    from paper_2507_14959_b200 import binding
    with pytest.raises(binding.PolymorphError) as e:
        binding.Linear(np.zeros((64, 64), np.float32), np.zeros(64, np.float32), max_adapters=256, max_rank=1 << 24, max_set=1, max_frames=1, tokens=1)
    assert e.value.code == binding.PM_ERR_OOM


@pytest.mark.parametrize("queries,keys,form", [(1, 9000, ("16 rows", True)), (256, 8000, ("tcgen05", True)), (40, 40, ("16 rows", False)), (1000, 1000, ("tcgen05", False))])
def test_attention_after_a_call_that_failed(queries, keys, form):
    """The error of an earlier call is not taken for this one's: all of its kernels run, the one that joins the parts too."""
    from paper_2507_14959_b200 import binding
    heads, kv_heads, dim = 8, 2, 128
    q, k, v = normal(1, queries, heads, dim).bfloat16().cuda(), normal(2, keys, kv_heads, dim).bfloat16().cuda(), normal(3, keys, kv_heads, dim).bfloat16().cuda()
    out, q_off, k_off = torch.full_like(q, 7.0), ints([0, queries]), ints([0, keys])
    took = binding.attention_packed_kernel(heads=heads, kv_heads=kv_heads, head_dim=dim, n_seqs=1, max_q=queries, max_kv=keys, workspace_bytes=1 << 28)
    assert (took[0], took[2] > 1) == form
    for before in (lambda: None, fail_a_call):                # the first call sets up what later ones find
        before()
        out.fill_(7.0)
        binding.attention_packed(q, k, v, out, q_off, queries, keys, 0, kv_offsets=k_off, causal=True)
    torch.cuda.synchronize()
    want, mean, size = expected(q, k, v, True, dim ** -0.5)
    assert ((out.double() - want).abs() <= bound(0, want, mean, size, dim, keys)).all()


def test_other_operators_after_a_call_that_failed():
    from paper_2507_14959_b200 import binding
    x, table, positions, gamma = normal(1, 50, 4, 64).bfloat16().cuda(), binding.RopeTable(64), ints(list(range(50))), torch.ones(64, device="cuda")
    f, off = x.float(), ints([0, 50])
    weights, rows, qkv = torch.ones(256, device="cuda"), x.flatten(1).contiguous(), normal(2, 50, 3 * 64).bfloat16().cuda()
    for like, call in ((x, lambda y: binding.rope(x, y, positions, table, 0)),
                       (x, lambda y: binding.qk_norm_rope(x, None, y, None, gamma, None, norm="rms", eps=1e-6, dtype=0)),
                       (f, lambda y: binding.attention_packed(f, f, f, y, off, 50, 50, 1)),
                       (rows, lambda y: binding.layernorm(rows, weights, weights, y, 1e-6, 0)),
                       (qkv[:, :64].contiguous(), lambda y: binding.attention(qkv, y, 1, 50, 1, 0))):
        before, after = torch.zeros_like(like), torch.zeros_like(like)
        call(before)
        fail_a_call()
        call(after)
        torch.cuda.synchronize()
        assert torch.equal(before, after) and before.abs().sum() > 0


@pytest.mark.parametrize("dtype,queries,keys,form", [(0, 3, 40, ("16 rows", 1)), (0, 2000, 2000, ("tcgen05", 1)), (0, 2, 9000, ("16 rows", 2)), (0, 256, 8000, ("tcgen05", 2)),
                                                     (1, 3, 40, ("fp32", 1)), (1, 70, 70, ("fp32", 1))])
def test_skipped_sequences_are_reported_without_a_status_word(dtype, queries, keys, form):
    from paper_2507_14959_b200 import binding
    heads, kv_heads, dim = 8, 2, 128
    t = (torch.bfloat16, torch.float32)[dtype]
    took = binding.attention_packed_kernel(heads=heads, kv_heads=kv_heads, head_dim=dim, n_seqs=1, max_q=queries, max_kv=keys, dtype=dtype,
                                           workspace_bytes=1 << 28 if form[1] > 1 else 0)
    assert took[0] == form[0] and (took[2] > 1) == (form[1] > 1)
    q, k, v = normal(1, queries, heads, dim).to(t).cuda(), normal(2, keys, kv_heads, dim).to(t).cuda(), normal(3, keys, kv_heads, dim).to(t).cuda()
    q_off, k_off, good, bad, status = ints([0, queries]), ints([0]), ints([keys]), ints([keys + 1]), ints([0])
    other = torch.cuda.Stream()

    def call(lengths, **more):
        out = torch.full_like(q, 7.0)
        torch.cuda.synchronize()
        binding.attention_packed(q, k, v, out, q_off, queries, keys, dtype, kv_offsets=k_off, kv_lengths=lengths, causal=True, **more)
        return out
    assert binding.operators_status() == 0
    call(good)
    assert binding.operators_status() == 0
    for stream in (None, other):
        out = call(bad, stream=stream)
        assert binding.operators_status(stream) == binding.PM_ERR_ARG and (out == 7).all()
        assert binding.operators_status(stream) == 0                       # taken away
    call(bad)                                              # a call that goes well does not clear what an earlier one has left
    call(good)
    assert binding.operators_status() == binding.PM_ERR_ARG
    call(bad, status=status)                               # a word of the caller's own is all that is written
    assert binding.operators_status() == 0 and status.item() == binding.PM_ERR_ARG


@pytest.mark.parametrize("dim,heads,kv_heads,lengths", [(128, 8, 2, [(256, 8000)]), (64, 4, 4, [(3000, 8192), (0, 500), (257, 0), (5, 5000)]), (64, 6, 2, [(700, 9000), (90, 300)]),
                                                        (128, 2, 2, [(2000, 5000)])])
def test_units_that_share_their_keys_without_causal_order(dim, heads, kv_heads, lengths):
    from paper_2507_14959_b200 import binding
    form = binding.attention_packed_kernel(heads=heads, kv_heads=kv_heads, head_dim=dim, n_seqs=len(lengths), max_q=max(a for a, _ in lengths), causal=False,
                                           max_kv=max(b for _, b in lengths), q_rows=sum(a for a, _ in lengths) + 3, kv_rows=sum(b for _, b in lengths) + 3,
                                           workspace_bytes=1 << 28)
    assert form[0] == "tcgen05" and form[2] > 1, form
    check(0, dim, heads, kv_heads, lengths, False, seed=73)


@pytest.mark.parametrize("n,seqs,heads", [(300, 4, 8), (100, 16, 8), (1000, 1, 12)])
def test_the_order_decides_the_kernel(n, seqs, heads):
    """Of the same sizes the causal call takes tiles of 16 rows, the full one units of 256."""
    from paper_2507_14959_b200 import binding
    for causal, kernel in ((True, "16 rows"), (False, "tcgen05")):
        assert binding.attention_packed_kernel(heads=heads, kv_heads=heads, head_dim=64, n_seqs=seqs, max_q=n, max_kv=n, q_rows=seqs * n + 3, kv_rows=seqs * n + 3,
                                               causal=causal)[0] == kernel
        check(0, 64, heads, heads, [(n, n)] * seqs, causal, packed=True, seed=74)


@pytest.mark.parametrize("dim,interleaved,axes", [(64, True, 1), (128, False, 1), (256, True, 2), (48, False, 2)])
@pytest.mark.parametrize("far", [100, 10 ** 6, 2 ** 31 - 1])
def test_angles_in_32_bits(dim, interleaved, axes, far):
    """Sine and cosine themselves: every pair is (1, 0).  Against the wrapped 64-bit products of the positions and the table's steps."""
    from paper_2507_14959_b200 import binding
    rows = 3000
    table = binding.RopeTable(dim, base=10000.0, interleaved=interleaved, axes=axes)
    at = torch.randint(-far, far, (rows, axes), generator=torch.Generator().manual_seed(dim), dtype=torch.int64)
    at[0], at[1] = far, 0
    step = np.array(table.table.step[:dim // 2], dtype=np.uint64)
    which = np.repeat(np.arange(axes), dim // 2 // axes)
    fraction = at.numpy().astype(np.uint64)[:, which] * step                  # of 2^64 to a turn, wrapped
    turns = torch.from_numpy((fraction >> np.uint64(11)).astype(np.float64) * 2.0 ** -53)
    first, second = (slice(0, dim, 2), slice(1, dim, 2)) if interleaved else (slice(0, dim // 2), slice(dim // 2, dim))
    x = torch.zeros((rows, 1, dim), device="cuda")
    x[..., first] = 1
    y = torch.zeros_like(x)
    binding.rope(x, y, at.int().cuda() if axes == 2 else at[:, 0].int().cuda(), table, 1)
    y = y[:, 0].cpu().double()
    # the angle's rounding to 2^-33 turns; to a float, 2^-24 of its distance from the nearest quarter turn; sine and cosine to a unit of
    # their last place, 2^-23 of them; the products with 1 and 0 are exact
    rest = (turns - torch.round(turns * 4) / 4).abs() * 2 * np.pi
    angle = 2 * np.pi * 2.0 ** -33 + 2.0 ** -24 * rest
    for got, want in ((y[:, first], torch.cos(2 * np.pi * turns)), (y[:, second], torch.sin(2 * np.pi * turns))):
        # (turns from 53 bits and the comparison's own roundings: 2^-50)
        excess = (got - want).abs() - (angle + 2.0 ** -23 * want.abs() + 2.0 ** -50)
        assert (excess <= 0).all(), excess.max()


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 1, 64), (16, 4, 128)])
def test_many_streams_with_histories_of_every_length(heads, kv_heads, dim):
    """More streams than a warp has lanes, in causal order; between the keys that their units see lie wide gaps."""
    from paper_2507_14959_b200 import binding
    lengths = [(n, n + kept) for n, kept in zip([300, 1, 40, 0, 129, 64, 600] * 11, [0, 9000, 3, 500, 0, 2000, 16, 0, 30000, 0, 700] * 7)]
    form = binding.attention_packed_kernel(heads=heads, kv_heads=kv_heads, head_dim=dim, n_seqs=len(lengths), max_q=600, max_kv=max(b for _, b in lengths),
                                           q_rows=sum(a for a, _ in lengths) + 3, kv_rows=sum(b for _, b in lengths) + 3)
    assert form[0] == "tcgen05" and len(lengths) > 64
    check(0, dim, heads, kv_heads, lengths, True, seed=75)


def test_one_more_stream_costs_about_one_more_stream():
    """A long history among short ones, with 32 streams and with 40: the search for the next unit does not go through all the keys between them."""
    from paper_2507_14959_b200 import binding
    heads, dim, new, kept = 64, 64, 16, 200000
    times, cache = {}, torch.randn((kept + 40 * new, 1, dim), device="cuda").bfloat16()
    for n in (32, 40):
        q = normal(n, n * new, heads, dim).bfloat16().cuda()
        out, q_off = torch.zeros_like(q), ints([i * new for i in range(n + 1)])
        lengths = [kept] + [new] * (n - 1)
        k_off, status = ints(np.cumsum([0] + lengths).tolist()), ints([0])
        at = []
        for _ in range(7):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            binding.attention_packed(q, cache, cache, out, q_off, new, kept, 0, kv_offsets=k_off, causal=True, status=status)
            end.record()
            torch.cuda.synchronize()
            at.append(start.elapsed_time(end))
        times[n] = sorted(at)[3]
        assert status.item() == 0
        want, mean, size = expected(q[:new], cache[:kept], cache[:kept], True, dim ** -0.5)
        assert ((out[:new].double() - want).abs() <= bound(0, want, mean, size, dim, kept)).all()
    assert times[40] < 3 * times[32], times               # level by level of 4 keys it was 20 times as long


@pytest.mark.parametrize("dtype", [0, 1])
def test_lists_of_a_call_without_rows_are_checked(dtype):
    """A limit, or a buffer, of no queries: sequences that have some are reported, whatever else is in order; nothing is written."""
    from paper_2507_14959_b200 import binding
    t = (torch.bfloat16, torch.float32)[dtype]
    q, empty = torch.ones((8, 2, 64), dtype=t, device="cuda"), torch.ones((0, 2, 64), dtype=t, device="cuda")
    out, status = torch.full_like(q, 7.0), ints([9])

    def call(rows, q_offsets, max_q, **keys):
        binding.attention_packed(rows, q, q, out[:len(rows)], ints(q_offsets), max_q, 8, dtype, status=status, **{n: ints(v) for n, v in keys.items()})
        return status.item()
    for rows, max_q in ((q, 0), (empty, 0), (empty, 5)):
        assert call(rows, [0, 0, 0], max_q) == 0
        assert call(rows, [0, 4, 4], max_q) == binding.PM_ERR_ARG
        assert call(rows, [0, 0, 0], max_q, kv_offsets=[0, 4, 8]) == 0
        assert call(rows, [0, 0, 0], max_q, kv_offsets=[0, 4, 9]) == binding.PM_ERR_ARG
        assert call(rows, [0] * 301, max_q, kv_offsets=[0] * 300, kv_lengths=[0] * 299 + [-1]) == binding.PM_ERR_ARG
        assert call(rows, [0], max_q) == 0
    assert (out == 7).all()


def test_missing_tensors_are_refused():
    from paper_2507_14959_b200 import binding
    x, off, gamma, table = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda"), ints([0, 4]), torch.ones(64, device="cuda"), binding.RopeTable(64)
    norm = lambda *a, **k: binding.qk_norm_rope(*a, norm="rms", eps=1e-6, dtype=0, **k)  # noqa: E731
    calls = [lambda i=i: binding.attention_packed(*[None if j == i else t for j, t in enumerate((x, x, x, x))], off, 4, 4, 0) for i in range(4)]
    calls += [lambda: binding.attention_packed(x, x, x, x, None, 4, 4, 0), lambda: binding.attention_packed(x, x, x, x, ints([]), 4, 4, 0)]
    calls += [lambda: binding.rope(None, x, off, table, 0), lambda: binding.rope(x, None, off, table, 0), lambda: binding.rope(x, x, None, table, 0),
              lambda: norm(None, x, x, x, gamma, gamma), lambda: norm(x, x, None, x, gamma, gamma), lambda: norm(x, x, x, None, gamma, gamma),
              lambda: norm(x, x, x, x, None, gamma), lambda: norm(x, x, x, x, gamma, None), lambda: norm(x, x, x, x, gamma, gamma, table=table),
              lambda: norm(x, x, x, x, gamma, gamma, positions=off)]
    for i, call in enumerate(calls):
        with pytest.raises(binding.PolymorphError) as e:
            call()
        assert e.value.code == binding.PM_ERR_ARG, i


def test_first_calls_in_32_bits_may_be_captured():
    """As in 16 bits: nothing is set up by a first call that a capture could not hold, and the replay computes what an eager call does."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2507_14959_b200 import binding
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
x = torch.randn(600, 8, 64, device="cuda")
table, at, g1 = binding.RopeTable(64), ints(list(range(600))), torch.ones(64, device="cuda")
few, all_, hist = ints([0, 3]), ints([0, 100, 600]), ints([0, 600])
def calls(o):
    binding.rope(x, o[0], at, table, 1)
    binding.qk_norm_rope(x, None, o[1], None, g1, None, norm="layer", eps=1e-6, dtype=1, positions=at, table=table)
    binding.attention_packed(x, x, x, o[2], few, 3, 600, 1, kv_offsets=hist, causal=True)
    binding.attention_packed(x, x, x, o[3], all_, 500, 500, 1)
outs, eager = ([torch.zeros_like(x) for _ in range(4)] for _ in range(2))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls(outs)
assert all(o.abs().sum() == 0 for o in outs)
graph.replay()
torch.cuda.synchronize()
calls(eager)
torch.cuda.synchronize()
assert all(torch.equal(a, b) and a[:3].abs().sum() > 0 for a, b in zip(outs, eager))
assert all(o[599].abs().sum() > 0 for o in (outs[0], outs[1], outs[3])) and outs[2][3:].abs().sum() == 0
print("captured")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "captured" in done.stdout, done.stderr[-2000:]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lengths,form", [([(1, 9000)], ("16 rows", True)), ([(256, 8000)], ("tcgen05", True)), ([(300, 300), (1000, 1000), (5, 700)] * 4, ("tcgen05", False)),
                                          ([(40, 40), (3, 500)], ("16 rows", False))])
def test_the_same_call_gives_the_same_bits(lengths, form, dim):
    """Every form, with other work in between: no sum's order depends on the run."""
    from paper_2507_14959_b200 import binding
    heads, kv_heads = 8, 2
    n_q, n_k = [a for a, _ in lengths], [b for _, b in lengths]
    took = binding.attention_packed_kernel(heads=heads, kv_heads=kv_heads, head_dim=dim, n_seqs=len(lengths), max_q=max(n_q), max_kv=max(n_k), q_rows=sum(n_q),
                                           kv_rows=sum(n_k), workspace_bytes=1 << 28)
    assert (took[0], took[2] > 1) == form, took
    q, k, v = (normal(i, n, h, dim).bfloat16().cuda() for i, n, h in ((1, sum(n_q), heads), (2, sum(n_k), kv_heads), (3, sum(n_k), kv_heads)))
    q_off, k_off, first = ints(np.cumsum([0] + n_q).tolist()), ints(np.cumsum([0] + n_k).tolist()), None
    noise, other = torch.randn(2048, 2048, device="cuda"), torch.cuda.Stream()
    for turn in range(8):
        out = torch.full_like(q, 7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            for _ in range(turn):
                noise @ noise
        binding.attention_packed(q, k, v, out, q_off, max(n_q), max(n_k), 0, kv_offsets=k_off, causal=True)
        torch.cuda.synchronize()
        first = out if first is None else first
        assert torch.equal(first, out)


def test_smoke_takes_no_cooperative_launch(capsys, monkeypatch):
    """smoke() is run under a profiler too, which the whole-network kernel's cooperative launch of clusters does not survive."""
    import __graft_entry__
    from paper_2507_14959_b200 import binding
    switched = []
    turn = binding.Model.set_small_batch_kernel
    monkeypatch.setattr(binding.Model, "set_small_batch_kernel", lambda m, on: (switched.append(bool(on)), turn(m, on))[1])
    __graft_entry__.smoke()
    said = capsys.readouterr().out
    # the whole-network kernel is one launch for the forward, the selection another
    assert switched == [False] and int(said.split("launches ")[1].split()[0]) > 20 and "packed sequences" in said


@pytest.mark.parametrize("dtype,queries,kernel", [(0, 1, "16 rows"), (0, 300, "tcgen05"), (1, 2, "fp32")])
def test_the_longest_history(dtype, queries, kernel):
    """2^24 equal weights add up exactly, whatever their order; a longer history is not served."""
    from paper_2507_14959_b200 import binding
    t, n, dim = (torch.bfloat16, torch.float32)[dtype], 1 << 24, 64
    form = binding.attention_packed_kernel(heads=8, kv_heads=1, head_dim=dim, n_seqs=1, max_q=queries, max_kv=2 ** 31 - 1, kv_rows=n + 1, dtype=dtype,
                                           workspace_bytes=1 << 28)
    assert form[0] == kernel
    q, k, v = normal(1, queries, 8, dim).to(t).cuda(), torch.zeros((n + 1, 1, dim), dtype=t, device="cuda"), torch.ones((n + 1, 1, dim), dtype=t, device="cuda")
    for keys in (n, n + 1):
        out, status = torch.full_like(q, 7.0), ints([5])
        binding.attention_packed(q, k, v, out, ints([0, queries]), queries, 2 ** 31 - 1, dtype, kv_offsets=ints([0]), kv_lengths=ints([keys]), causal=True,
                                 status=status)
        assert status.item() == (0 if keys == n else binding.PM_ERR_ARG)
        assert (out == (1 if keys == n else 7)).all()
