"""Packed caches: what outputs owe to the rows that a query sees, and to nothing else, against 64 bits on the GPU.

An output of bf16 is a number near the exact one, rounded: its rounding alone is 2^-8 / sqrt(3) of it at most in the mean square
(an error even over a step that is 2^-7 of the power of two below the value), 2.26e-3.  Where weights go through fp16, once or twice,
each adds 2^-11 / sqrt(3) of the value at most, 2.8e-4, independent from row to row.  Together 2.3e-3: DIGITS allows 2.5e-3.
"""
import threading

import pytest
import torch

import paper_2412_05693_b200 as bm
from tests import packed_reference as ref
from tests.test_packed_gpu import DT, ints, make, same

pytestmark = pytest.mark.gpu
DIGITS = 2.5e-3


def exact(q, k, v, lens, first, scale):
    """The attention in 64 bits over what k and v are packed as; q (b, I, Hq, d), k and v (b, n, Hkv, d)."""
    b, I, Hq, d = q.shape
    n, Hkv = k.shape[1:3]
    k, v = (ref.packed_values(x).cuda().repeat_interleave(Hq // Hkv, 2) for x in (k, v))
    row, query = torch.arange(n, device="cuda"), torch.arange(I, device="cuda")
    seen = (row < (ints(lens)[:, None] - (I - 1 - query))[..., None]) & (row >= ints(first)[:, None, None])
    k, v = (torch.where(seen.any(1)[..., None, None], x, 0.0) for x in (k, v))
    logits = torch.einsum("bihd,bnhd->bhin", q.double(), k) * scale
    seen = seen[:, None].expand_as(logits)
    p = torch.where(seen.any(-1, keepdim=True), logits.masked_fill(~seen, -torch.inf).softmax(-1), 0.0)
    return torch.einsum("bhin,bnhd->bihd", p, v)


def normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_far_below_zero_read_as_zeros(dtype):
    gen = torch.Generator("cuda").manual_seed(1)
    lens = [-2 ** 31, -2 ** 31 + 40, -1, 2 ** 31 - 1, 50]
    cache = make(5, 2, 2, 64, 100, dtype)
    k = normal(gen, 5, 100, 2, 64).to(DT[dtype])
    cache.write(k, -k)
    for row0, rows in ((0, 100), (40, 60), (65, 35), (99, 1)):
        for got, x in zip(cache.read(row0, rows, lens=ints(lens)), (k, -k)):
            want = ref.packed_values(x)[:, row0:row0 + rows]
            want[:3] = 0
            want[4, max(0, 50 - row0):] = 0
            same(got, want)


def hidden_rows(b, Hq, Hkv, d, I, dtype, path):
    """Rows behind the length or before the first row change nothing, however large: not the outputs' digits, not one bit."""
    gen = torch.Generator("cuda").manual_seed(2)
    n, lens, first = 200, [137, 200, 130, 165], [5, 67, 0, 31]
    lens, first = [lens[s % 4] for s in range(b)], [first[s % 4] for s in range(b)]
    row = torch.arange(n, device="cuda")
    visible = ((row < ints(lens)[:, None]) & (row >= ints(first)[:, None]))[..., None, None]
    k, v = normal(gen, b, n, Hkv, d) * 1e-4, normal(gen, b, n, Hkv, d) * 1e-4
    q = (normal(gen, b, I, Hq, d) * 1e4).to(DT[dtype])
    outs = []
    for hidden in (0.0, 1.0, 5e5, 3e38):
        kh, vh = (torch.where(visible, x, hidden * torch.sign(x)).to(DT[dtype]) for x in (k, v))
        cache = make(b, Hq, Hkv, d, n, dtype, queries_max=I)
        cache.write(kh, vh)
        outs.append(cache.attend(q, ints(lens), first=ints(first)))
        assert bm.last_packed_path() == path
    want = exact(q, k.to(DT[dtype]), v.to(DT[dtype]), lens, first, d ** -0.5)
    allowed = DIGITS if dtype == "bf16" else 2.0 ** -18
    assert max((o.double() - want).norm() / want.norm() for o in outs) <= allowed
    assert all(torch.equal(o, outs[0]) for o in outs)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_not_seen_change_nothing_in_blocks(d):
    hidden_rows(40, 2, 2, d, 128, "bf16", 1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,I,dtype", [(4, 1, 1, "bf16"), (2, 2, 2, "bf16"), (8, 1, 1, "bf16"), (4, 2, 7, "bf16"), (4, 2, 1, "f32"), (2, 2, 9, "f32")])
def test_rows_that_are_not_seen_change_nothing(Hq, Hkv, I, dtype, d):
    hidden_rows(4, Hq, Hkv, d, I, dtype, 0)


SHAPES = [(2, 1, 1, 1, 1000, 0), (2, 4, 1, 1, 1000, 0), (2, 2, 1, 2, 1000, 0), (2, 8, 1, 1, 1000, 0), (2, 4, 1, 6, 1000, 0), (40, 2, 2, 128, 400, 1)]


@pytest.mark.parametrize("r", [30.0, 100.0, 1000.0])
@pytest.mark.parametrize("b,Hq,Hkv,I,n,path", SHAPES)
def test_queries_with_an_outlier(b, Hq, Hkv, I, n, path, r):
    """One channel of the queries r times the others, and that channel of the keys an r-th: logits are as without, so their digits are
    those that the other channels keep beside the outlier.  Steps of 2^-21 of the outlier leave 1000 * 2^-21 / sqrt(12) of them, and of the
    logits, which have a deviation of 3, 5e-4."""
    gen = torch.Generator("cuda").manual_seed(3)
    q, k, v = normal(gen, b, I, Hq, 128), normal(gen, b, n, Hkv, 128), normal(gen, b, n, Hkv, 128)
    q[..., 5] *= r
    k[..., 5] /= r
    k[..., 40:] *= 4.0
    k[1::2, n - 77:] = v[1::2, n - 77:] = torch.nan      # (behind their samples' lengths)
    q, k, v = q.bfloat16(), k.bfloat16(), v.bfloat16()
    cache = make(b, Hq, Hkv, 128, n, "bf16", queries_max=I)
    cache.write(k, v)
    lens = [n, n - 77] * (b // 2)
    out = cache.attend(q, ints(lens))
    assert bm.last_packed_path() == path
    want = exact(q, k, v, lens, [0] * b, 128 ** -0.5)
    assert (out.double() - want).norm() <= DIGITS * want.norm()


@pytest.mark.parametrize("scale", [0.0, 0.35, 1.0])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,Hq,Hkv,I,n,path", [(4, 4, 4, 1, 1500, 0), (4, 8, 2, 1, 1500, 0), (4, 16, 2, 1, 1500, 0), (4, 8, 2, 2, 700, 0),
                                               (4, 10, 2, 3, 700, 0), (40, 2, 2, 128, 400, 1), (20, 8, 4, 150, 400, None)])
def test_outputs_are_the_rounded_exact_ones_but_for_few_digits(b, Hq, Hkv, I, n, path, d, scale):
    """Without the rounding of the outputs, errors are those of the weights: each is rounded to fp16 (a half step is 2^-12 to 2^-11 of it,
    2.0e-4 in the mean square), and outside of blocks once more with its row's scale: 2.9e-4 of an output where few rows make it up, less
    where many do.  Twice that is allowed, over at least 16 outputs' mean square.  (Logits' errors, 2^-18 of them at most, do not show.  A
    tile of values with 8 bits would leave 1.6e-3.)"""
    gen = torch.Generator("cuda").manual_seed(4)
    q, k, v = (normal(gen, b, t, h, d).bfloat16() for t, h in ((I, Hq), (n, Hkv), (n, Hkv)))
    cache = make(b, Hq, Hkv, d, n, "bf16", queries_max=I, softmax_scale=scale)
    cache.write(k, v)
    lens = [n, n - 77] * (b // 2)
    out, took = cache.attend(q, ints(lens)).double(), bm.last_packed_path()
    assert path in (took, None)
    want = exact(q, k, v, lens, [0] * b, scale or d ** -0.5)
    rounded = want.bfloat16().double()
    # errors of the outputs' rounding and of what is rounded are independent: their squares add up
    inner = (out - want).square().sum() - (rounded - want).square().sum()
    assert inner <= (4e-4 if took == 1 else 6e-4) ** 2 * want.square().sum()
    assert (out - want).norm() <= DIGITS * want.norm()


@pytest.mark.parametrize("Hq,Hkv,d,I", [(4, 4, 64, 1), (8, 2, 128, 1), (8, 1, 64, 3), (3, 3, 128, 9)])
def test_single_precision_has_its_digits_in_every_group(Hq, Hkv, d, I):
    """Groups of very different size: each has the digits that it has among its like, which are the same bits when sizes are powers of two."""
    gen = torch.Generator("cuda").manual_seed(5)
    n, scale = 4000, 4 * d ** -0.5
    q, k, v = normal(gen, 2, I, Hq, d), normal(gen, 2, n, Hkv, d), normal(gen, 2, n, Hkv, d)
    v[:, 500:] *= 3.0                      # (growing on the way)
    sizes = torch.tensor([2.0 ** -8, 2.0 ** 8, 2.0 ** -3, 1.0] if d == 128 else [2.0 ** 8, 2.0 ** -8], device="cuda").repeat_interleave(32)
    outs = []
    for by in (torch.ones_like(sizes), sizes):
        cache = make(2, Hq, Hkv, d, n, "f32", queries_max=I, softmax_scale=scale)
        cache.write(k, v * by)
        outs.append(cache.attend(q, ints([n, n - 100])))
    want = exact(q, k, v, [n, n - 100], [0, 0], scale)
    assert (outs[0].double() - want).norm() <= 2.0 ** -18 * want.norm()
    assert torch.equal(outs[1], outs[0] * sizes)


@pytest.mark.parametrize("Hq,I,dtype", [(4, 1, "bf16"), (8, 1, "bf16"), (2, 9, "bf16"), (4, 1, "f32")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** 26, 2.0 ** 121])
def test_logits_next_to_the_largest_number(size, Hq, I, dtype, d):
    """Queries of 2^121: their logits are numbers of 32 bits, and the row with the largest takes the whole weight."""
    gen = torch.Generator("cuda").manual_seed(6)
    n = 60
    q, k, v = (normal(gen, 1, I, Hq, d) * size).to(DT[dtype]), normal(gen, 1, n, 1, d).to(DT[dtype]), normal(gen, 1, n, 1, d).to(DT[dtype])
    q[0, 0, 0] = 0.0                       # (a mean over all rows)
    cache = make(1, Hq, 1, d, n, dtype, queries_max=I)
    cache.write(k, v)
    out = cache.attend(q, ints([n]))
    want = exact(q, k, v, [n], [0], d ** -0.5)
    assert out.isfinite().all()
    assert (out.double() - want).norm() <= (DIGITS if dtype == "bf16" else 2.0 ** -18) * want.norm()


@pytest.mark.parametrize("Hq,I,dtype", [(4, 1, "bf16"), (8, 1, "bf16"), (4, 1, "f32"), (2, 9, "f32")])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 18, 2.0 ** 23, 2.0 ** 26, 2.0 ** 100])
def test_equal_logits_of_any_size(size, Hq, I, dtype):
    """Rows with one key share the weight evenly, also where their values' scales change on the way and the logit leaves no room for them."""
    gen = torch.Generator("cuda").manual_seed(10)
    n, d = 700, 128
    q, k = (normal(gen, 1, I, Hq, d) * size).to(DT[dtype]), normal(gen, 1, 1, 1, d).expand(1, n, 1, d).to(DT[dtype])
    v = (normal(gen, 1, n, 1, d) + 1.0) * 2.0 ** (torch.arange(n, device="cuda") // 50)[:, None, None]
    v = v.to(DT[dtype])
    cache = make(1, Hq, 1, d, n, dtype, queries_max=I)
    cache.write(k.contiguous(), v)
    out = cache.attend(q, ints([n]))
    want = exact(torch.zeros_like(q), k, v, [n], [0], 1.0)
    assert (out.double() - want).norm() <= (DIGITS if dtype == "bf16" else 2.0 ** -18) * want.norm()


@pytest.mark.parametrize("size", [2.0 ** 26, 2.0 ** 121])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_next_to_the_largest_number_in_blocks(d, size):
    gen = torch.Generator("cuda").manual_seed(9)
    b, I, n = 40, 128, 300
    q, k, v = (normal(gen, b, I, 2, d) * size).bfloat16(), normal(gen, b, n, 2, d).bfloat16(), normal(gen, b, n, 2, d).bfloat16()
    q[:, 3] = 0.0
    cache = make(b, 2, 2, d, n, "bf16", queries_max=I)
    cache.write(k, v)
    lens = [300, 270] * 20
    out = cache.attend(q, ints(lens))
    assert bm.last_packed_path() == 1
    want = exact(q, k, v, lens, [0] * b, d ** -0.5)
    assert out.isfinite().all()
    assert (out.double() - want).norm() <= DIGITS * want.norm()


def test_handles_that_take_fewer_samples_per_call_are_packed_at_once():
    """How many samples a call of the evicting handle may have is a matter of its workspace, which packing does not use; so is how far each
    sample is in its sequence of the pairs' positions."""
    gen = torch.Generator("cuda").manual_seed(7)
    handle = bm.BatchMaxCache(bm.Config(batch=5, n_q_heads=4, n_kv_heads=2, head_dim=64, kv_max=40, block_max=40, max_call_samples=2))
    rows = [[normal(gen, ns, 40, h, 64).bfloat16() for h in (4, 2, 2)] for ns in (2, 2, 1)]
    for i, (q, k, v) in enumerate(rows):
        handle.prefill_block(q, k, v, 0, sample0=2 * i)
    cache = make(5, 4, 2, 64, 64, "bf16")
    assert cache.write_from(handle) == 40
    gk, gv = cache.read(0, 40)
    same(gk, ref.packed_values(torch.cat([r[1] for r in rows])))
    same(gv, ref.packed_values(torch.cat([r[2] for r in rows])))
    q, k, v = (normal(gen, 2, 24, h, 64).bfloat16() for h in (4, 2, 2))
    handle.prefill_block(q, k, v, 40, sample0=2, evict_to=40)                      # samples 2 and 3 go on
    assert cache.write_from(handle) == 40
    for s in range(5):
        for h in range(2):
            _, _, kr, vr = handle.export(sample=s, kv_head=h, rows=True)
            same(cache.read(0, 40)[0][s, :, h], ref.packed_values(kr))
            same(cache.read(0, 40)[1][s, :, h], ref.packed_values(vr))
    with pytest.raises(bm.BMError) as e:   # samples that the handle does not have
        make(6, 4, 2, 64, 64, "bf16").write_from(handle)
    assert e.value.code == 1


def test_one_cache_used_by_several_threads():
    gen = torch.Generator("cuda").manual_seed(8)
    cache = make(2, 8, 2, 128, 600, "bf16")
    k, v = normal(gen, 2, 600, 2, 128).bfloat16(), normal(gen, 2, 600, 2, 128).bfloat16()
    cache.write(k, v)
    lens = ints([600, 431])
    q = [normal(gen, 2, 1, 8, 128).bfloat16() for _ in range(4)]
    want = [cache.attend(x, lens) for x in q]
    spaces, streams = [cache.new_workspace() for _ in q], [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    calls, bad, go = 1500, [], threading.Barrier(len(q))

    def work(i):
        with torch.cuda.stream(streams[i]):
            out = torch.empty_like(q[i])
            go.wait()
            for _ in range(calls):
                cache.attend(q[i], lens, out=out, workspace=spaces[i])
            streams[i].synchronize()
            if not torch.equal(out, want[i]):
                bad.append(i)

    before = bm.kernel_launch_count()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(q))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
    assert bm.kernel_launch_count() - before == 2 * calls * len(q)   # the attention, and the joining of its shares


def test_rows_beyond_the_cache_are_refused_before_memory_is_taken():
    cache = make(2, 2, 2, 64, 100, "bf16")
    cache.read(0, 1)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    held = torch.cuda.memory_allocated()
    for args, kw in [((0, 2 ** 31 - 1), {}), ((1, 2 ** 31 - 1), {}), ((2 ** 31 - 1, 2 ** 31 - 1), {}), ((0, 10 ** 7), dict(stream=torch.cuda.current_stream())),
                     ((0, 10 ** 7), dict(lens=ints([1, 1]))), ((0, 100), dict(nsamples=10 ** 6)), ((0, 100), dict(nsamples=-1)),
                     ((0, 100), dict(sample0=3)), ((0, 0), {}), ((0, -5), {}), ((2 ** 40, 1), {})]:
        with pytest.raises(bm.BMError) as e:
            cache.read(*args, **kw)
        assert e.value.code == 1
    assert torch.cuda.max_memory_allocated() <= held + 4096


def test_a_wait_that_runs_out_is_reported_and_harms_nothing():
    gen = torch.Generator("cuda").manual_seed(11)
    cache = make(2, 4, 2, 64, 100, "bf16")
    k, q, lens = normal(gen, 2, 100, 2, 64).bfloat16(), normal(gen, 2, 1, 4, 64).bfloat16(), ints([100, 60])
    cache.write(k, k)
    want = cache.attend(q, lens)
    cache.selftest_wait_timeout()
    assert cache.status() == 6
    cache.clear_status()
    assert torch.equal(cache.attend(q, lens), want) and cache.status() == 0
