"""Packed caches on the GPU: written, read back, and attended to, against the format and the attention in 64 bits."""
import math

import pytest
import torch

import paper_2412_05693_b200 as bm
from tests import packed_reference as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(b, Hq, Hkv, d, capacity, dtype, **kw):
    return bm.PackedCache(bm.PackedConfig(batch=b, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, capacity=capacity, dtype=dtype, **kw))


def rows(gen, *shape, dtype, spread=1.0):
    x = torch.randn(*shape, generator=gen) * spread
    x[..., 3::29] *= 6.0
    return x.to(DT[dtype]).cuda()


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def same(got, want):
    """Bit for bit up to the sign of zeros; NaN where NaN is wanted."""
    want = want.to(got.dtype)
    got = got.cpu()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))


# ---- write, read ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,Hkv,d,I", [(1, 1, 64, 1), (3, 2, 128, 5), (2, 5, 64, 33), (4, 8, 128, 130), (7, 3, 64, 1)])
def test_rows_read_back_as_the_format_says(b, Hkv, d, I, dtype):
    gen = torch.Generator().manual_seed(b * 1000 + I)
    k, v = rows(gen, b, I, Hkv, d, dtype=dtype), rows(gen, b, I, Hkv, d, dtype=dtype, spread=0.01)
    cache = make(b, Hkv, Hkv, d, I + 3, dtype)
    cache.write(k, v)
    gk, gv = cache.read(0, I + 3)
    same(gk[:, :I], ref.packed_values(k))
    same(gv[:, :I], ref.packed_values(v))
    assert not gk[:, I:].any() and not gv[:, I:].any()
    assert cache.status() == 0


def test_ties_peaks_of_both_signs_and_extremes():
    """Exact ties of x / s, equal peaks of opposite signs, saturation, subnormal scales, zeros, NaN and infinities."""
    x = torch.zeros(16, 128)
    half = torch.arange(32) - 16
    x[0, :32] = half / 2.0                                # peak -8 -> s = 1: every other element a tie
    x[0, 32:64] = half / 2.0 + 0.5                        # peak -7.5
    x[1, :32] = torch.tensor([4.0, -4.0] * 16)            # equal magnitudes: the first one is at -8
    x[1, 32:64] = torch.tensor([-4.0, 4.0] * 16)
    x[2, 5], x[2, 40] = 3e38, -3e38                       # scales saturate
    x[3, 0], x[3, 1] = 1e-7, 3e-8                         # a subnormal scale
    x[3, 33] = 1e-12                                      # a scale of zero
    x[4, 7] = math.nan
    x[4, 100] = math.inf
    x[5, 64] = -math.inf
    x[6] = 1.0
    x[7] = torch.linspace(-1, 1, 128)
    x[8, :32] = -8.0 + half * 0.0625
    x[9] = 65504.0 * 8
    x[10, :32] = (half * 0.5).flip(0)                     # peak +8 comes last: the first largest magnitude is 7.5's -> -8 order
    x[11, 0], x[11, 1:32] = -8.0, torch.arange(31) * 0.25 + 2.0 ** -17
    x[12, 0], x[12, 1:32] = -8.0, torch.arange(31) * 0.25 - 2.0 ** -17
    for dtype in ("bf16", "f32"):
        for d in (64, 128):
            t = x.to(DT[dtype]).view(1, -1, 1, d).cuda()
            cache = make(1, 1, 1, d, t.shape[1], dtype)
            cache.write(t, -t)
            gk, gv = cache.read(0, t.shape[1])
            same(gk, ref.packed_values(t))
            same(gv, ref.packed_values(-t))


def test_quotients_next_to_ties_in_single_precision():
    """x one or two steps of fp32 away from every (k + 1/2) s, for many scales."""
    gen = torch.Generator().manual_seed(5)
    peaks = (torch.rand(4096, generator=gen) + 0.5) * torch.tensor([1.0, -1.0]).repeat(2048) * 2.0 ** torch.randint(-8, 8, (4096,), generator=gen)
    s = (peaks / -8).half().float()
    x = torch.empty(4096, 32)
    x[:, 0] = peaks
    for j in range(1, 32):
        t = (j % 15 - 7.5) * s
        steps = j // 15 - 1
        for _ in range(abs(steps)):
            t = torch.nextafter(t, torch.full_like(t, math.inf * steps))
        x[:, j] = torch.where(t.abs() < peaks.abs(), t, 0.0)
    x = x.view(1, 2048, 1, 64).cuda()
    cache = make(1, 1, 1, 64, 2048, "f32")
    cache.write(x, x)
    gk, gv = cache.read(0, 2048)
    same(gk, ref.packed_values(x))
    same(gv, ref.packed_values(x))


def test_ragged_starts_counts_and_rows_that_stay():
    b, Hkv, d, I, cap = 5, 3, 128, 7, 40
    gen = torch.Generator().manual_seed(2)
    cache = make(b, Hkv, Hkv, d, cap, "bf16")
    old = rows(gen, b, cap, Hkv, d, dtype="bf16"), rows(gen, b, cap, Hkv, d, dtype="bf16")
    cache.write(*old)
    k, v = rows(gen, b, I, Hkv, d, dtype="bf16"), rows(gen, b, I, Hkv, d, dtype="bf16")
    start, counts = [0, 33, 12, 5, 39], [7, 7, 0, 3, 1]
    cache.write(k, v, start=ints(start), counts=ints(counts))
    want = [ref.packed_values(t).clone() for t in old]
    for s in range(b):
        for w, t in zip(want, (k, v)):
            w[s, start[s]:start[s] + counts[s]] = ref.packed_values(t[s, :counts[s]])
    for got, w in zip(cache.read(0, cap), want):
        same(got, w)
    lens = [40, 0, 1, 17, 39]
    for got, w in zip(cache.read(4, 20, lens=ints(lens)), want):
        w = w[:, 4:24].clone()
        for s in range(b):
            w[s, max(0, lens[s] - 4):] = 0
        same(got, w)
    assert cache.status() == 0


def test_rows_outside_the_cache_are_not_stored_and_reported():
    cache = make(3, 2, 2, 64, 10, "bf16")
    gen = torch.Generator().manual_seed(3)
    k = rows(gen, 3, 4, 2, 64, dtype="bf16")
    cache.write(k, k, start=ints([8, -2, 2 ** 31 - 2]))
    want = torch.zeros(3, 10, 2, 64, dtype=torch.float64)
    want[0, 8:] = ref.packed_values(k[0, :2])
    want[1, :2] = ref.packed_values(k[1, 2:])
    for got in cache.read(0, 10):
        same(got, want)
    assert cache.status() == 3
    cache.clear_status()
    assert cache.status() == 0


def test_strided_rows_layers_and_sample_ranges():
    b, Hq, Hkv, d, I, L = 4, 4, 2, 64, 6, 3
    gen = torch.Generator().manual_seed(4)
    cache = make(b, Hq, Hkv, d, 16, "f32", n_layers=L)
    qkv = rows(gen, 2, 2 * I, Hq + 2 * Hkv, d, dtype="f32")[:, ::2]
    k, v = qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    cache.write(k, v, start=ints([3, 9]), layer=1, sample0=1)
    for layer in range(L):
        want = [torch.zeros(b, 16, Hkv, d, dtype=torch.float64) for _ in range(2)]
        if layer == 1:
            for w, t in zip(want, (k, v)):
                w[1, 3:9], w[2, 9:15] = ref.packed_values(t[0]), ref.packed_values(t[1])
        for got, w in zip(cache.read(0, 16, layer=layer), want):
            same(got, w)
    got = cache.read(3, 6, layer=1, sample0=1, nsamples=1)
    same(got[0], ref.packed_values(k[:1]))


@pytest.mark.parametrize("dtype,compaction", [("bf16", "stable"), ("f32", "stable"), ("bf16", "fill")])
def test_the_pairs_that_a_prefill_kept_are_packed(dtype, compaction):
    b, Hq, Hkv, d, K = 3, 4, 2, 64, 48
    gen = torch.Generator().manual_seed(6)
    handle = bm.BatchMaxCache(bm.Config(batch=b, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, kv_max=K, block_max=32, dtype=dtype,
                                        compaction=compaction, n_layers=2))
    for layer in range(2):
        for pos in range(0, 128, 32):
            q, k, v = (rows(gen, b, 32, h, d, dtype=dtype) for h in (Hq, Hkv, Hkv))
            handle.prefill_block(q, k, v, pos, evict_to=K, layer=layer)
    cache = make(b, Hq, Hkv, d, K + 5, dtype)
    assert cache.write_from(handle, from_layer=1) == K
    gk, gv = cache.read(0, K + 5)
    for s in range(b):
        for h in range(Hkv):
            _, _, kr, vr = handle.export(layer=1, sample=s, kv_head=h, rows=True)
            same(gk[s, :K, h], ref.packed_values(kr))
            same(gv[s, :K, h], ref.packed_values(vr))
    assert not gk[:, K:].any()
    # a range of its samples into another place
    one = make(b, Hq, Hkv, d, K, dtype)
    one.write_from(handle, sample0=2, nsamples=1, from_layer=1, from_sample0=0)
    assert torch.equal(one.read(0, K, sample0=2)[0], gk[:1, :K]) and not one.read(0, K, nsamples=2)[0].any()


def test_a_handle_fed_from_the_host_is_packed_between_its_calls():
    """Host-fed calls run on the handle's own streams: those before a packing are read complete, those after wait for it."""
    b, Hq, Hkv, d, K, I = 4, 8, 4, 128, 512, 512
    gen = torch.Generator().manual_seed(40)
    cfg = dict(batch=b, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, kv_max=K, block_max=I)
    host = [[(torch.randn(b, I, h, d, generator=gen)).bfloat16().pin_memory() for h in (Hq, Hkv, Hkv)] for _ in range(4)]
    want = []
    for fed in (False, True):
        handle, caches = bm.BatchMaxCache(bm.Config(**cfg)), [make(b, Hq, Hkv, d, K, "bf16") for _ in range(4)]
        for i, (q, k, v) in enumerate(host):
            if fed:
                handle.prefill_block_host(q, k, v, i * I, torch.empty_like(q).pin_memory(), evict_to=K)
            else:
                handle.prefill_block(q.cuda(), k.cuda(), v.cuda(), i * I, evict_to=K)
                torch.cuda.synchronize()
            caches[i].write_from(handle)
            if not fed:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        got = [torch.stack(c.read(0, K)) for c in caches]
        if fed:
            assert all(torch.equal(a, w) for a, w in zip(got, want))
        want = got
        handle.close()


def test_kernels_of_packed_caches_are_timed():
    cache = make(1, 2, 1, 64, 40, "bf16")
    gen = torch.Generator().manual_seed(41)
    k, q = rows(gen, 1, 40, 1, 64, dtype="bf16"), rows(gen, 1, 1, 2, 64, dtype="bf16")
    lens = ints([40])

    def calls():
        cache.write(k, k)
        cache.read(0, 40)
        cache.attend(q, lens)

    calls()
    ms, launches = bm.binding.profile_pass(calls)["packed"]
    assert launches == 4 and ms > 0 and "packed" not in bm.binding.profile_pass(lambda: None)


# ---- attend -----------------------------------------------------------------------------------------------------------------
def check_attend(b, Hq, Hkv, d, I, capacity, lens, first, dtype, seed=0, spread=1.0, scale=0.0, split=0, cache=None):
    blocks = dtype == "bf16" and I * (Hq // Hkv) > 64       # many query rows may go through fp16 tiles
    gen = torch.Generator().manual_seed(seed)
    k, v = rows(gen, b, capacity, Hkv, d, dtype=dtype), rows(gen, b, capacity, Hkv, d, dtype=dtype, spread=spread)
    q = rows(gen, b, I, Hq, d, dtype=dtype)
    cache = cache or make(b, Hq, Hkv, d, capacity, dtype, queries_max=I, softmax_scale=scale)
    cache.write(k, v)
    out = cache.attend(q, ints(lens), first=ints(first) if first is not None else None, max_len=split)
    want, wide, slack = ref.attend(q.double().cpu(), ref.packed_values(k), ref.packed_values(v), lens, first or [0] * b,
                                   scale or d ** -0.5, DT[dtype], blocks)
    allowed = ref.bound(want, wide, slack, DT[dtype], capacity, float(v.double().abs().max()), blocks)
    err = (out.double().cpu() - want).abs()
    assert not out.isnan().any()
    assert (err <= allowed).all(), f"worst error / allowed: {(err / allowed).max():.3f}, largest error {err.max():.3e}"
    seen_none = [[max(0, min(n, capacity)) - (I - 1 - i) <= f for i in range(I)] for n, f in zip(lens, first or [0] * b)]
    for s in range(b):
        for i in range(I):
            if seen_none[s][i]:
                assert not out[s, i].any()
    assert cache.status() == 0
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (4, 2), (8, 2), (8, 1), (6, 2), (12, 1)])
def test_one_token(Hq, Hkv, d, dtype):
    check_attend(4, Hq, Hkv, d, 1, 300, [300, 1, 0, 171], None, dtype, seed=Hq * 10 + Hkv)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1025])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_around_the_tiles(n, dtype):
    check_attend(2, 4, 2, 128, 1, n, [n, n - 1], None, dtype, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("I,Hq,Hkv", [(2, 4, 2), (3, 8, 1), (5, 5, 1), (8, 8, 2), (17, 4, 4), (40, 4, 1)])
def test_several_queries_are_causal(I, Hq, Hkv, dtype):
    lens = [150, I, max(I - 2, 0), 64 + I // 2, 149]
    check_attend(5, Hq, Hkv, 64, I, 150, lens, None, dtype, seed=I)
    check_attend(5, Hq, Hkv, 128, I, 150, lens, [0, 0, 0, 64, 33], dtype, seed=I + 100)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,I,Hq,Hkv,path", [(3, 65, 1, 1, 0), (40, 113, 2, 2, 1), (40, 128, 2, 2, 1), (40, 129, 2, 2, 1), (40, 256, 2, 2, 1),
                                             (60, 257, 2, 2, 1), (40, 60, 4, 2, 1), (40, 40, 6, 2, 1), (40, 17, 24, 2, 1), (20, 300, 8, 4, 1),
                                             (140, 8, 12, 1, 1), (2, 300, 8, 4, 0)])
def test_blocks_of_queries(b, I, Hq, Hkv, path, d):
    n = 400
    for lens, first in (([n, I, 333], None), ([n - 1, I + 1, max(I - 3, 1), 0, 2 * I, 277], [130, 0, 0, 5, 128, 1])):
        lens, first = [lens[s % len(lens)] for s in range(b)], first and [first[s % len(first)] for s in range(b)]
        check_attend(b, Hq, Hkv, d, I, n, lens, first, "bf16", seed=I)
        assert bm.last_packed_path() == path


@pytest.mark.parametrize("spread", [1e-6, 1e-3, 100.0, 30000.0])
def test_blocks_of_queries_over_values_of_any_size(spread):
    check_attend(64, 2, 2, 128, 70, 200, [200, 77] * 32, None, "bf16", spread=spread, seed=31)
    assert bm.last_packed_path() == 1


def test_blocks_over_long_caches():
    for d in (64, 128):
        check_attend(1, 128, 128, d, 120, 3000, [2999], [100], "bf16", seed=33)
        assert bm.last_packed_path() == 1
        check_attend(1, 2, 1, d, 70, 3000, [2999], [100], "bf16", seed=34)


@pytest.mark.parametrize("copies,path", [(1, 0), (20, 1)])
def test_blocks_meet_rows_that_are_not_finite(copies, path):
    b, Hq, Hkv, d, I, n = 3, 2, 2, 128, 130, 300
    gen = torch.Generator().manual_seed(34)
    k, v, q = (rows(gen, b, t, h, d, dtype="bf16") for t, h in ((n, Hkv), (n, Hkv), (I, Hq)))
    v[0, 200, 0, 40] = math.nan                       # group 1, head 0: queries that see row 200
    v[0, 260, 0, 41] = -math.inf                      # (a later one in the same group)
    k[1, 250, 1, 0] = math.inf                        # head 1: queries that see row 250
    k[2, 290:], v[2, 290:] = math.nan, math.inf       # behind sample 2's length
    k[2, :7], v[2, :7] = -math.inf, math.nan          # before its first row
    q[2, 5, 1, 3] = math.nan
    k, v, q = (t.repeat(copies, 1, 1, 1) for t in (k, v, q))
    cache = make(b * copies, Hq, Hkv, d, n, "bf16", queries_max=I)
    cache.write(k, v)
    out = cache.attend(q, ints([300, 300, 290] * copies), first=ints([0, 0, 7] * copies)).float().cpu()
    assert bm.last_packed_path() == path
    bad = torch.zeros(b, I, Hq, d, dtype=torch.bool)
    bad[0, I - 99 - 1:, 0, 32:64] = True              # query i sees rows below 300 - (129 - i): row 200 from i = 30 on
    bad[1, I - 49 - 1:, 1] = True
    bad[2, 5, 1] = True
    assert torch.equal(out.isnan(), bad.repeat(copies, 1, 1, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_left_padding_and_lengths_outside_the_cache(dtype):
    check_attend(7, 4, 2, 64, 1, 96, [96, 96, 96, 1000, -5, 40, 40], [0, 95, 96, 31, 0, 41, -7], dtype, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread", [1e-6, 1e-3, 100.0, 30000.0])
def test_values_of_any_size(dtype, spread):
    check_attend(2, 4, 2, 128, 1, 200, [200, 77], None, dtype, spread=spread, seed=11)


@pytest.mark.parametrize("split", [0, 1, 100, 4096])
def test_results_do_not_need_the_right_longest_length(split):
    check_attend(2, 8, 2, 128, 1, 4096, [4096, 2000], None, "bf16", split=split, seed=12)


def test_values_that_grow_along_the_cache():
    """Scales that rise and fall by far more than the kernel's normalisation spans at once."""
    for dtype in ("bf16", "f32"):
        gen = torch.Generator().manual_seed(13)
        b, H, d, n = 2, 2, 64, 320
        k, v, q = (rows(gen, b, t, H, d, dtype=dtype) for t in (n, n, 1))
        size = 2.0 ** (torch.arange(n) % 160 / 6.0 - 12)
        v = (v.float() * size.cuda()[None, :, None, None]).to(DT[dtype])
        v[..., 32:] = (v[..., 32:].float() * 1e-3).to(DT[dtype])
        cache = make(b, H, H, d, n, dtype)
        cache.write(k, v)
        out = cache.attend(q, ints([n, n - 9]))
        pv = ref.packed_values(v)
        want, wide, slack = ref.attend(q.double().cpu(), ref.packed_values(k), pv, [n, n - 9], [0, 0], d ** -0.5, DT[dtype])
        # a group's smallest weights are fp16 numbers next to its largest scale: that group's largest value counts
        vmax = pv.abs().view(b, n, H, d // 32, 32).amax((1, 4)).repeat_interleave(32, -1)[:, None]
        allowed = ref.bound(want, wide, slack, DT[dtype], n, vmax)
        assert ((out.double().cpu() - want).abs() <= allowed).all()


def test_not_finite_rows_reach_the_queries_that_see_them_and_no_others():
    for dtype in ("bf16", "f32"):
        b, Hq, Hkv, d, I, n = 4, 4, 2, 128, 3, 100
        gen = torch.Generator().manual_seed(14)
        k, v, q = rows(gen, b, n, Hkv, d, dtype=dtype), rows(gen, b, n, Hkv, d, dtype=dtype), rows(gen, b, I, Hq, d, dtype=dtype)
        v[0, 97, 0, 40] = math.nan         # group 1 of sample 0, head 0: the last row but two
        k[1, 98, 1, 0] = math.inf          # sample 1, head 1: seen by the last two queries
        k[2, 99], v[2, 99] = math.nan, math.inf    # behind sample 2's length
        k[3, :7], v[3, :7] = -math.inf, math.nan   # before sample 3's first row
        cache = make(b, Hq, Hkv, d, n, dtype, queries_max=I)
        cache.write(k, v)
        out = cache.attend(q, ints([100, 100, 99, 100]), first=ints([0, 0, 0, 7])).float().cpu()
        bad = torch.zeros(b, I, Hq, d, dtype=torch.bool)
        bad[0, :, :2, 32:64] = True        # rows < 98, < 99, < 100: every query sees row 97
        bad[1, 1:, 2:] = True
        assert torch.equal(out.isnan(), bad)


def test_queries_that_are_not_finite_or_zero():
    cache = make(1, 4, 1, 64, 50, "bf16")
    gen = torch.Generator().manual_seed(15)
    k, v, q = rows(gen, 1, 50, 1, 64, dtype="bf16"), rows(gen, 1, 50, 1, 64, dtype="bf16"), rows(gen, 1, 1, 4, 64, dtype="bf16")
    cache.write(k, v)
    q[0, 0, 1, 3] = math.nan
    q[0, 0, 2] = 0.0
    q[0, 0, 3] *= 1e-30
    out = cache.attend(q, ints([50])).float().cpu()
    assert out[0, 0, 1].isnan().all() and not out[0, 0, [0, 2, 3]].isnan().any()
    mean = ref.packed_values(v)[0, :, 0].mean(0)
    wide = ref.packed_values(v)[0, :, 0].abs().mean(0)
    assert ((out[0, 0, 2:] - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -9 * wide).all()
    # one that sees no row has a row of zeros all the same; the others of its tile are not touched by it
    for dtype, bad in [("bf16", math.nan), ("bf16", math.inf), ("f32", math.nan)]:
        cache = make(1, 1, 1, 64, 50, dtype, queries_max=4)
        k, v, q = (rows(gen, 1, n, 1, 64, dtype=dtype) for n in (50, 50, 4))
        cache.write(k, v)
        q[0, 0, 0, 1] = q[0, 2, 0, 9] = bad
        out = cache.attend(q, ints([40]), first=ints([38])).float().cpu()     # rows 38 .. 36, 37, 38 and 39
        assert not out[0, :2].any() and out[0, 2].isnan().all() and not out[0, 3].isnan().any()


def test_a_long_cache_whose_offsets_pass_32_bits():
    """The caches' code bytes pass 2^32: the last layer's last sample still is its own."""
    b, Hkv, d, n, L = 2, 8, 128, 65536, 70          # 70 * 2 * 8 * 65536 * 64 bytes of key codes
    cache = make(b, 8, Hkv, d, n, "bf16", n_layers=L)
    gen = torch.Generator().manual_seed(16)
    k, v, q = rows(gen, 1, 40, Hkv, d, dtype="bf16"), rows(gen, 1, 40, Hkv, d, dtype="bf16"), rows(gen, 1, 1, 8, d, dtype="bf16")
    cache.write(k, v, start=ints([n - 40]), layer=L - 1, sample0=1)
    same(cache.read(n - 40, 40, layer=L - 1, sample0=1)[0], ref.packed_values(k))
    out = cache.attend(q, ints([n]), first=ints([n - 40]), layer=L - 1, sample0=1)
    want, wide, slack = ref.attend(q.double().cpu(), ref.packed_values(k), ref.packed_values(v), [40], [0], d ** -0.5, torch.bfloat16)
    assert ((out.double().cpu() - want).abs() <= ref.bound(want, wide, slack, torch.bfloat16, 40, 30.0)).all()
    assert not cache.read(n - 40, 40, layer=L - 1, nsamples=1)[0].any() and not cache.read(0, 40, layer=0)[0].any()


def test_strided_queries_ranges_and_given_outputs():
    b, Hq, Hkv, d, n = 4, 6, 2, 64, 70
    gen = torch.Generator().manual_seed(17)
    cache = make(b, Hq, Hkv, d, n, "bf16", queries_max=2)
    k, v = rows(gen, b, n, Hkv, d, dtype="bf16"), rows(gen, b, n, Hkv, d, dtype="bf16")
    cache.write(k, v)
    qkv = rows(gen, b, 2, Hq + 4, d, dtype="bf16")
    q = qkv[:, :, :Hq]
    lens = ints([70, 69, 3, 50])
    whole = cache.attend(q.contiguous(), lens)
    assert torch.equal(cache.attend(q, lens), whole)
    out = torch.full((2, 2, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    assert cache.attend(q[1:3], lens[1:3], out=out, sample0=1) is out
    want, wide, slack = ref.attend(q[1:3].double().cpu(), ref.packed_values(k[1:3]), ref.packed_values(v[1:3]), [69, 3], [0, 0], d ** -0.5, torch.bfloat16)
    assert ((out.double().cpu() - want).abs() <= ref.bound(want, wide, slack, torch.bfloat16, n, 30.0)).all()


def test_other_streams_with_a_workspace_each():
    gen = torch.Generator().manual_seed(18)
    cache = make(2, 8, 2, 128, 2048, "bf16")
    k, v = rows(gen, 2, 2048, 2, 128, dtype="bf16"), rows(gen, 2, 2048, 2, 128, dtype="bf16")
    cache.write(k, v)
    q = [rows(gen, 2, 1, 8, 128, dtype="bf16") for _ in range(2)]
    lens = ints([2048, 1500])
    want = [cache.attend(x, lens) for x in q]
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [cache.new_workspace() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            got[i].append(cache.attend(q[i], lens, stream=streams[i], workspace=spaces[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_a_captured_step_replayed_as_the_caches_grow():
    """Write, then attend, as one graph: the lengths move on the device between replays."""
    b, Hq, Hkv, d, n0, steps = 3, 8, 2, 64, 60, 10
    gen = torch.Generator().manual_seed(19)
    cache = make(b, Hq, Hkv, d, n0 + steps, "bf16")
    k, v = rows(gen, b, n0 + steps, Hkv, d, dtype="bf16"), rows(gen, b, n0 + steps, Hkv, d, dtype="bf16")
    qs = rows(gen, steps, b, 1, Hq, d, dtype="bf16")
    cache.write(k[:, :n0], v[:, :n0])
    lens, q = ints([n0, n0 - 7, 1]), torch.empty(b, 1, Hq, d, dtype=torch.bfloat16, device="cuda")
    kt, vt = torch.empty(b, 1, Hkv, d, dtype=torch.bfloat16, device="cuda"), torch.empty(b, 1, Hkv, d, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)

    def step():
        cache.write(kt, vt, start=lens)
        lens.add_(1)
        cache.attend(q, lens, out=out)

    kt.copy_(k[:, :1]); vt.copy_(v[:, :1]); q.copy_(qs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    lens.copy_(ints([n0, n0 - 7, 1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    start = [n0, n0 - 7, 1]
    held = [(k[s, :start[s]].clone(), v[s, :start[s]].clone()) for s in range(b)]
    for t in range(steps):
        kt.copy_(k[:, n0 + t:n0 + t + 1]); vt.copy_(v[:, n0 + t:n0 + t + 1]); q.copy_(qs[t])
        graph.replay()
        for s in range(b):
            held[s] = torch.cat([held[s][0], kt[s]]), torch.cat([held[s][1], vt[s]])
            want, wide, slack = ref.attend(q[s:s + 1].double().cpu(), ref.packed_values(held[s][0])[None], ref.packed_values(held[s][1])[None],
                                           [start[s] + t + 1], [0], d ** -0.5, torch.bfloat16)
            allowed = ref.bound(want, wide, slack, torch.bfloat16, n0 + steps, 30.0)
            assert ((out[s:s + 1].double().cpu() - want).abs() <= allowed).all()
    assert cache.status() == 0


def test_a_captured_block_gives_what_an_eager_one_gives():
    gen = torch.Generator().manual_seed(35)
    cache = make(20, 4, 2, 128, 600, "bf16", queries_max=150)
    cache.write(rows(gen, 20, 600, 2, 128, dtype="bf16"), rows(gen, 20, 600, 2, 128, dtype="bf16"))
    q, lens = rows(gen, 20, 150, 4, 128, dtype="bf16"), ints([600, 480] * 10)
    want = cache.attend(q, lens)
    assert bm.last_packed_path() == 1
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(q, lens, out=out)
    for n in ([600, 480], [333, 600]):
        lens.copy_(ints(n * 10))
        graph.replay()
        assert torch.equal(out, want if n[0] == 600 else cache.attend(q, lens))


def test_same_results_from_run_to_run():
    gen = torch.Generator().manual_seed(20)
    for Hq, Hkv, I, n in ((32, 8, 1, 5000), (8, 8, 1, 700), (8, 2, 9, 300), (80, 40, 200, 500)):
        cache = make(2, Hq, Hkv, 128, n, "bf16", queries_max=I)
        cache.write(rows(gen, 2, n, Hkv, 128, dtype="bf16"), rows(gen, 2, n, Hkv, 128, dtype="bf16"))
        q, lens = rows(gen, 2, I, Hq, 128, dtype="bf16"), ints([n, n - 5])
        first = cache.attend(q, lens)
        assert all(torch.equal(cache.attend(q, lens), first) for _ in range(5))


@pytest.mark.parametrize("b", [33, 64, 65, 1024, 2500])
def test_many_samples_of_unequal_length(b):
    """A warp finds its run among the samples' tiles: every lane has several samples, or more than fit one look."""
    gen = torch.Generator().manual_seed(b)
    lens = torch.randint(0, 71, (b,), generator=gen).tolist()
    lens[3:9] = [0] * 6
    check_attend(b, 2, 1, 64, 1, 70, lens, None, "bf16", seed=b)
    check_attend(b, 1, 1, 64, 1, 70, [0] * (b - 1) + [70], None, "f32", seed=b)


@pytest.mark.parametrize("b,Hq,I,path", [(3, 4, 1, 0), (40, 8, 64, 1)])
def test_nothing_to_see(b, Hq, I, path):
    cache = make(b, Hq, 2, 64, 200, "bf16", queries_max=I)
    gen = torch.Generator().manual_seed(50)
    cache.write(rows(gen, b, 200, 2, 64, dtype="bf16"), rows(gen, b, 200, 2, 64, dtype="bf16"))
    q = rows(gen, b, I, Hq, 64, dtype="bf16")
    for lens, first in (([0] * b, None), ([-3] * b, [5] * b), ([150] * b, [150] * b), ([200] * b, [2 ** 31 - 1] * b)):
        out = torch.full_like(q, 7.0)
        cache.attend(q, ints(lens), first=None if first is None else ints(first), out=out)
        assert not out.any() and bm.last_packed_path() == path


@pytest.mark.parametrize("Hq,Hkv,d,I", [(4, 4, 64, 1), (8, 2, 128, 1), (8, 1, 64, 3)])
def test_single_precision_has_all_its_digits(Hq, Hkv, d, I):
    """The worst case that `bound` allows would hide a lost second half of a query or a weight (2^-12 of it, 1e-4 of the outputs): fp32
    steps of logits up to 32 and of their sums leave a few 2^-20."""
    gen = torch.Generator().manual_seed(55)
    n = 900
    k, v, q = (torch.randn(2, t, h, d, generator=gen).cuda() for t, h in ((n, Hkv), (n, Hkv), (I, Hq)))
    cache = make(2, Hq, Hkv, d, n, "f32", queries_max=I)
    cache.write(k, v)
    out = cache.attend(q, ints([n, n - 100])).double().cpu()
    want, _, _ = ref.attend(q.double().cpu(), ref.packed_values(k), ref.packed_values(v), [n, n - 100], [0, 0], d ** -0.5, torch.float32)
    assert (out - want).norm() <= 2.0 ** -18 * want.norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-3, 0.7, 6.0])
def test_flat_and_peaked_weights(scale, dtype):
    check_attend(2, 8, 2, 64, 1, 500, [500, 333], None, dtype, seed=51, scale=scale)
    check_attend(2, 4, 2, 128, 2, 500, [500, 333], None, dtype, seed=52, scale=scale)


def test_what_a_workspace_holds_before_does_not_matter():
    gen = torch.Generator().manual_seed(53)
    for b, Hq, Hkv, I in ((3, 8, 2, 1), (30, 8, 4, 64)):
        cache = make(b, Hq, Hkv, 128, 700, "bf16", queries_max=I)
        cache.write(rows(gen, b, 700, Hkv, 128, dtype="bf16"), rows(gen, b, 700, Hkv, 128, dtype="bf16"))
        q, lens = rows(gen, b, I, Hq, 128, dtype="bf16"), ints([700, 0, 650] * (b // 3))
        cache.workspace.zero_()
        want = cache.attend(q, lens)
        for byte in (0xff, 0x7f, 0x01):
            cache.workspace.fill_(byte)
            assert torch.equal(cache.attend(q, lens), want)


def test_repeated_rows_counts_beyond_the_tokens_and_closed_caches():
    gen = torch.Generator().manual_seed(54)
    cache = make(3, 2, 2, 64, 70, "bf16")
    k, v = rows(gen, 1, 40, 2, 64, dtype="bf16"), rows(gen, 3, 1, 2, 64, dtype="bf16")
    cache.write(k.expand(3, -1, -1, -1), v.expand(-1, 40, -1, -1), start=ints([0, 30, 5]), counts=ints([1000, 40, -1]))
    gk, gv = cache.read(0, 70)
    wk, wv = ref.packed_values(k[0]), ref.packed_values(v)
    same(gk[0, :40], wk)
    same(gv[1, 30:], wv[1].expand(40, -1, -1))
    assert not gk[0, 40:].any() and not gk[1, :30].any() and not gk[2].any() and cache.status() == 0
    cache.close()
    for call in (lambda: cache.read(0, 1), lambda: cache.write(v, v), lambda: cache.status()):
        with pytest.raises(bm.BMError) as e:
            call()
        assert e.value.code == 1


# ---- together ---------------------------------------------------------------------------------------------------------------
def test_prefill_with_eviction_then_decoding_over_packed_caches():
    """A prompt through an evicting handle, its kept pairs packed, tokens decoded over 4 bits."""
    b, Hq, Hkv, d, K, steps = 2, 8, 2, 128, 128, 6
    gen = torch.Generator().manual_seed(21)
    handle = bm.BatchMaxCache(bm.Config(batch=b, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, kv_max=K, block_max=128))
    for pos in range(0, 512, 128):
        handle.prefill_block(*(rows(gen, b, 128, h, d, dtype="bf16") for h in (Hq, Hkv, Hkv)), pos, evict_to=K)
    cache = make(b, Hq, Hkv, d, K + steps, "bf16")
    n = cache.write_from(handle)
    pairs = [[torch.stack([handle.export(sample=s, kv_head=h, rows=True)[i] for h in range(Hkv)], 1) for i in (2, 3)] for s in range(b)]
    handle.close()
    lens = ints([n] * b)
    for _ in range(steps):
        q, k, v = (rows(gen, b, 1, h, d, dtype="bf16") for h in (Hq, Hkv, Hkv))
        cache.write(k, v, start=lens)
        lens += 1
        out = cache.attend(q, lens)
        for s in range(b):
            pairs[s] = [torch.cat([pairs[s][0], k[s].cpu()]), torch.cat([pairs[s][1], v[s].cpu()])]
        pk, pv = (ref.packed_values(torch.stack([pairs[s][i] for s in range(b)])) for i in range(2))
        want, wide, slack = ref.attend(q.double().cpu(), pk, pv, lens.tolist(), [0] * b, d ** -0.5, torch.bfloat16)
        assert ((out.double().cpu() - want).abs() <= ref.bound(want, wide, slack, torch.bfloat16, K + steps, 30.0)).all()
    assert cache.status() == 0


# ---- refusals ---------------------------------------------------------------------------------------------------------------
def test_refused_calls_leave_the_caches_alone():
    cache = make(2, 4, 2, 64, 20, "bf16", queries_max=2)
    gen = torch.Generator().manual_seed(22)
    k = rows(gen, 2, 4, 2, 64, dtype="bf16")
    q = rows(gen, 2, 1, 4, 64, dtype="bf16")
    lens = ints([4, 4])
    for call, code in [
        (lambda: cache.write(k, k, layer=1), 1), (lambda: cache.write(k, k, sample0=1), 1), (lambda: cache.write(k, k, sample0=-1), 1),
        (lambda: cache.read(0, 21), 1), (lambda: cache.read(-1, 2), 1), (lambda: cache.read(20, 1), 1),
        (lambda: cache.attend(rows(gen, 2, 3, 4, 64, dtype="bf16"), lens), 1), (lambda: cache.attend(q, lens, layer=-1), 1),
        (lambda: cache.attend(q, lens, max_len=-1), 1),
        (lambda: cache.attend(q, lens, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), 2),
        (lambda: cache.write(rows(gen, 2, 21, 2, 64, dtype="bf16"), rows(gen, 2, 21, 2, 64, dtype="bf16")), 1),
    ]:
        with pytest.raises(bm.BMError) as e:
            call()
        assert e.value.code == code
    odd = torch.zeros(2 * 4 * 2 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    for call in [
        lambda: cache.write(k.float(), k.float()), lambda: cache.write(k, k[:, :3]), lambda: cache.write(k.cpu(), k.cpu()),
        lambda: cache.write(k[..., ::2], k[..., ::2]), lambda: cache.write(k, k, start=torch.zeros(2, dtype=torch.int64, device="cuda")),
        lambda: cache.write(k, k, start=ints([1])), lambda: cache.attend(q, lens.cpu()), lambda: cache.attend(q[:, :, :2], lens),
        lambda: cache.attend(q, lens, out=torch.empty(2, 1, 4, 64, device="cuda")), lambda: cache.write(k[:, :0], k[:, :0]),
        lambda: cache.read(0, 2, out=(k, k)),
    ]:
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(bm.BMError):   # rows that do not start on 16 bytes
        cache.write(odd[1:1 + k.numel()].view_as(k), k)
    assert not cache.read(0, 20)[0].any() and cache.status() == 0


def test_refused_packing_of_handles():
    handle = bm.BatchMaxCache(bm.Config(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, kv_max=16, block_max=16, n_layers=2))
    gen = torch.Generator().manual_seed(23)
    handle.prefill_block(*(rows(gen, 1, 16, h, 64, dtype="bf16") for h in (4, 2, 2)), 0)
    for cache, kw, code in [(make(2, 4, 2, 64, 16, "bf16"), {}, 4),                                # unequal lengths
                            (make(2, 4, 2, 64, 15, "bf16"), dict(nsamples=1), 3), (make(2, 4, 2, 128, 16, "bf16"), dict(nsamples=1), 1),
                            (make(2, 4, 2, 64, 16, "f32"), dict(nsamples=1), 1), (make(2, 4, 4, 64, 16, "bf16"), dict(nsamples=1), 1),
                            (make(2, 4, 2, 64, 16, "bf16"), dict(nsamples=1, from_layer=2), 1)]:
        with pytest.raises(bm.BMError) as e:
            cache.write_from(handle, **kw)
        assert e.value.code == code
    empty = make(2, 4, 2, 64, 16, "bf16")
    assert empty.write_from(handle, from_layer=1) == 0 and not empty.read(0, 16)[0].any()
    padded = bm.BatchMaxCache(bm.Config(batch=1, n_q_heads=4, n_kv_heads=2, head_dim=64, kv_max=16, block_max=16))
    padded.set_left_pad([3])
    padded.prefill_block(*(rows(gen, 1, 16, h, 64, dtype="bf16") for h in (4, 2, 2)), 0)
    one = make(1, 4, 2, 64, 16, "bf16")
    with pytest.raises(bm.BMError) as e:
        one.write_from(padded)
    assert e.value.code == 4
    padded.evict(13)                       # padding leaves first: now the caches can be packed
    assert one.write_from(padded) == 13
