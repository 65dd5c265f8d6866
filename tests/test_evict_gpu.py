"""Attention weights added up per row and eviction by them, against the 64-bit statements of oracle/evict.py.

Eviction moves values: every byte has one right value.  Tolerances of the weights, relative L2 over the rows of one (sequence, KV head): a
rotated key or query channel is off by at most a few 2^-24 of itself, stepped over up to 32 rows (32 * 2 * 2^-24 = 4e-6); a score by
that share of the sum of its terms' magnitudes, 20 at most in these inputs in units of log2, and a weight by ln 2 times that:
6e-5.  Tolerance 1e-4.  Outputs as in test_attend_gpu: bf16 1e-2, fp32 2e-4."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import evict as oe
from paper_2505_00570_b200 import binding as fk
from paper_2505_00570_b200 import synth
from tests import parity

pytestmark = pytest.mark.gpu

WEIGHTS, OUT = 1e-4, {torch.float32: 2e-4, torch.bfloat16: 1e-2}


@pytest.fixture(scope="session", autouse=True)
def small_segment():
    """Holds one small segment of torch's allocator until the session ends.  A test that runs later in the session leaves less free memory
    than the 2 MB that a new segment takes, or a little more, by what else the process holds, and compares tensors then."""
    keep = torch.zeros(1, device="cuda")
    yield keep


@pytest.fixture(scope="module")
def ctx():
    c = fk.Context(0)
    yield c
    c.close()


def caches(B, L, H, cap, dtype, seed=1, hd=128):
    return synth.make_cache(synth.Workload("evict", B, L, H, hd, cap, dtype, 4, 0.9, 2, synth.BASE_SEED + seed), "cuda")


def queries(shape, dtype, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def masses(shape, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.rand(shape, generator=gen, device="cuda")


# ---- decode attention that adds up its weights ----

def check_decode(ctx, k, v, layer, q, lens, base=10000.0, scale=0.0, heads=None):
    B, L, H, cap, _ = k.shape
    G = q.shape[1] // H
    mass = torch.zeros(B, L, H, cap, device="cuda")
    plain = ctx.attend_decode(k, v, layer, q, lens, rope_base=base, scale=scale)
    out = ctx.attend_decode_mass(k, v, layer, q, mass, lens, rope_base=base, scale=scale)
    assert ctx.last_device_status() == fk.OK
    for b, h in heads or np.ndindex(B, H):
        kk, vv, qq = (parity.to_f64(x) for x in (k[b, layer, h], v[b, layer, h], q[b, h * G:(h + 1) * G]))
        want = oe.weights(qq[:, None], kk, lens[b], base, None if scale <= 0 else scale)
        got = parity.to_f64(mass[b, layer, h])
        assert parity.rel_l2(got[:lens[b]], want) <= WEIGHTS
        assert not got[lens[b]:].any()
        o = oa.attend_decode(qq, kk, vv, lens[b], base, None if scale <= 0 else scale)
        for g in range(G):
            assert parity.rel_l2(parity.to_f64(out[b, h * G + g]), o[g]) <= OUT[k.dtype]
    rest = mass.clone()
    rest[:, layer] = 0
    assert not bool(rest.any())                                   # other layers keep their values
    assert float((out.float() - plain.float()).norm() / plain.float().norm()) <= 2 * OUT[k.dtype]
    return out, mass


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_decode_mass_small_all_heads(ctx, dtype, G):
    k, v = caches(3, 3, 2, 300, dtype)
    k0, v0 = k.clone(), v.clone()
    check_decode(ctx, k, v, 1, queries((3, 2 * G, 128), dtype, 5 + G), [300, 37, 1])
    assert torch.equal(k, k0) and torch.equal(v, v0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("G", [1, 4])
def test_decode_mass_lengths_around_tiles_and_splits(ctx, dtype, G):
    w = synth.Workload("evict", 1, 1, 2, 128, 1100, dtype, 4, 0.9, 2, synth.BASE_SEED + 13)
    (_, k), (_, v) = parity.guarded_cache(w, torch.device("cuda"), fill_len=1100, row_pad=8)
    q = queries((1, 2 * G, 128), dtype, 6)
    for n in (1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 191, 192, 193, 255, 257, 511, 512, 513, 1023, 1025, 1100):
        check_decode(ctx, k, v, 0, q, [n], heads=[(0, 1)])


@pytest.mark.parametrize("base,scale", [(0.0, 0.0), (500000.0, 0.05), (10000.0, 0.1)])
def test_decode_mass_rope_off_other_base_and_scale(ctx, base, scale):
    for dtype in (torch.bfloat16, torch.float32):
        k, v = caches(2, 2, 3, 200, dtype, 12)
        check_decode(ctx, k, v, 0, queries((2, 6, 128), dtype, 3), [199, 64], base, scale)


def test_decode_mass_adds_up_and_is_the_same_every_time(ctx):
    k, v = caches(2, 2, 2, 2000, torch.bfloat16, 14)
    q = queries((2, 8, 128), torch.bfloat16, 4)
    start = masses((2, 2, 2, 2000), 3)
    a, b, zero = start.clone(), start.clone(), torch.zeros_like(start)
    ctx.attend_decode_mass(k, v, 1, q, zero, [2000, 777])
    for m in (a, b):
        for _ in range(3):
            out = ctx.attend_decode_mass(k, v, 1, q, m, [2000, 777])
    assert torch.equal(a, b)
    assert torch.allclose(a, start + 3 * zero, rtol=4 * 2 ** -23)
    assert torch.equal(a[:, 0], start[:, 0]) and torch.equal(a[1, 1, :, 777:], start[1, 1, :, 777:])
    assert torch.allclose(zero.sum(3)[:, 1].cpu(), torch.full((2, 2), 4.0), rtol=1e-5)   # every query head gives away one


def test_decode_mass_many_sequences_streams_and_capture(ctx):
    B = 130
    k, v = caches(B, 1, 1, 80, torch.bfloat16, 15)
    lens = [1 + (37 * b) % 80 for b in range(B)]
    q = queries((B, 2, 128), torch.bfloat16, 4)
    _, mass = check_decode(ctx, k, v, 0, q, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = torch.zeros_like(mass)
    with torch.cuda.stream(side):
        ctx.attend_decode_mass(k, v, 0, q, other, lens)
    side.synchronize()
    assert torch.equal(mass, other)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.attend_decode_mass(k, v, 0, q, other, lens, out=out)
    assert torch.equal(mass, other)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.allclose(other, 3 * mass, rtol=4 * 2 ** -23)


def test_decode_mass_rows_behind_the_last_may_hold_anything(ctx):
    k, v = caches(1, 1, 2, 300, torch.bfloat16, 16)
    q = queries((1, 4, 128), torch.bfloat16, 4)
    mass = torch.zeros(1, 1, 2, 300, device="cuda")
    out = ctx.attend_decode_mass(k, v, 0, q, mass, [211])
    k[..., 211:, :], v[..., 211:, :] = float("nan"), float("inf")
    again = torch.zeros_like(mass)
    again[..., 211:] = float("nan")
    assert torch.equal(out, ctx.attend_decode_mass(k, v, 0, q, again, [211]))
    assert torch.equal(mass[..., :211], again[..., :211]) and bool(again[..., 211:].isnan().all())


def test_decode_mass_refusals(ctx):
    k, v = caches(1, 2, 2, 64, torch.bfloat16, 17)
    q, mass = queries((1, 2, 128), torch.bfloat16, 4), torch.zeros(1, 2, 2, 64, device="cuda")
    for kw in ({"lens": [0]}, {"lens": [65]}, {"layer": 2}, {"scale": float("nan")}, {"mass": mass[..., :32]}, {"mass": mass.double()},
               {"mass": mass.cpu()}, {"out": q}, {"q": q.float()}):
        a = dict(k=k, v=v, layer=0, q=q, mass=mass, lens=[5]) | kw
        with pytest.raises(fk.FreqKVError):
            ctx.attend_decode_mass(**a)
    with pytest.raises(fk.FreqKVError) as e:
        ctx.attend_decode_mass(k, v, 0, queries((1, 6, 128), torch.bfloat16, 4), mass, [5])
    assert e.value.status == fk.ERR_UNSUPPORTED
    assert not bool(mass.any())


# ---- a chunk's weights ----

def check_chunk(ctx, k, layer, q, lens, base=10000.0, scale=0.0, heads=None):
    B, L, H, cap, _ = k.shape
    G, n = q.shape[1] // H, q.shape[2]
    start = masses((B, L, H, cap), 3) * 0.01
    mass = start.clone()
    ctx.attend_mass(k, layer, q, mass, lens, rope_base=base, scale=scale)
    assert ctx.last_device_status() == fk.OK
    for b, h in heads or np.ndindex(B, H):
        want = oe.weights(parity.to_f64(q[b, h * G:(h + 1) * G]), parity.to_f64(k[b, layer, h]), lens[b], base, None if scale <= 0 else scale)
        got = parity.to_f64(mass[b, layer, h, :lens[b]])
        assert parity.rel_l2(got, parity.to_f64(start[b, layer, h, :lens[b]]) + want) <= WEIGHTS
        assert torch.equal(mass[b, layer, h, lens[b]:], start[b, layer, h, lens[b]:])
    mass[:, layer] = start[:, layer]
    assert torch.equal(mass, start)


@pytest.mark.parametrize("G,n,lens", [(1, 1, [1, 70]), (2, 2, [2, 3]), (3, 64, [64, 200]), (4, 129, [129, 300]), (1, 200, [230, 299]),
                                      (9, 5, [65, 128]), (2, 127, [127, 255]), (1, 128, [128, 256]), (8, 17, [257, 300])])
def test_chunk_mass_small(ctx, G, n, lens):
    k, _ = caches(2, 2, 2, 300, torch.bfloat16, n)
    check_chunk(ctx, k, 1, queries((2, 2 * G, n, 128), torch.bfloat16, n), lens)


@pytest.mark.parametrize("base,scale", [(0.0, 0.0), (500000.0, 0.05)])
def test_chunk_mass_rope_off_other_base_and_scale(ctx, base, scale):
    k, _ = caches(1, 1, 2, 500, torch.bfloat16, 21)
    check_chunk(ctx, k, 0, queries((1, 4, 130, 128), torch.bfloat16, 3), [497], base, scale)


def test_chunk_mass_padded_rows_many_sequences_and_what_lies_behind(ctx):
    w = synth.Workload("evict", 1, 1, 2, 128, 700, torch.bfloat16, 4, 0.9, 2, synth.BASE_SEED + 13)
    (_, k), _ = parity.guarded_cache(w, torch.device("cuda"), fill_len=700, row_pad=8)
    q = queries((1, 2, 300, 128), torch.bfloat16, 6)
    check_chunk(ctx, k, 0, q, [600])
    a, b = torch.zeros(1, 1, 2, 700, device="cuda"), torch.zeros(1, 1, 2, 700, device="cuda")
    ctx.attend_mass(k, 0, q, a, [600])
    k[..., 600:, :] = float("nan")
    ctx.attend_mass(k, 0, q, b, [600])
    assert torch.equal(a, b)
    B = 130
    k, _ = caches(B, 1, 1, 40, torch.bfloat16, 15)
    check_chunk(ctx, k, 0, queries((B, 2, 3, 128), torch.bfloat16, 6), [3 + (11 * i) % 38 for i in range(B)])


def test_chunk_mass_of_one_token_is_that_of_decoding(ctx):
    k, v = caches(2, 1, 2, 1777, torch.bfloat16, 23)
    q = queries((2, 8, 128), torch.bfloat16, 4)
    a, b = torch.zeros(2, 1, 2, 1777, device="cuda"), torch.zeros(2, 1, 2, 1777, device="cuda")
    ctx.attend_decode_mass(k, v, 0, q, a, [1777, 5])
    ctx.attend_mass(k, 0, q.unsqueeze(2).contiguous(), b, [1777, 5])
    assert float((a - b).norm() / a.norm()) <= 2 * WEIGHTS


def test_chunk_mass_large_against_64_bits_on_the_gpu(ctx):
    """Many tiles a CTA: the weights of 1500 queries over 6000 rows, in 64-bit torch."""
    n, T = 1500, 6000
    k, _ = caches(1, 1, 2, T, torch.bfloat16, 24)
    q = queries((1, 6, n, 128), torch.bfloat16, 4)
    mass = torch.zeros(1, 1, 2, T, device="cuda")
    ctx.attend_mass(k, 0, q, mass, [T])
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       torch.arange(T, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(64, device="cuda").double() / 64))
    z = lambda x, at: torch.complex(x[..., :64].double(), x[..., 64:].double()) * at
    hidden = torch.full((n, T), -torch.inf, dtype=torch.float64, device="cuda").triu(T - n + 1)
    for h in range(2):
        s = (z(q[0, 3 * h:3 * h + 3], turn[T - n:]) @ z(k[0, 0, h], turn).conj().T).real / 128 ** 0.5 + hidden
        want = torch.softmax(s, -1).sum((0, 1))
        assert float((mass[0, 0, h].double() - want).norm() / want.norm()) <= 2e-5
        assert abs(float(mass[0, 0, h].double().sum()) / (3 * n) - 1) <= 2e-6


@pytest.mark.parametrize("n,G", [(2, 1), (3, 4), (5, 1)])
def test_chunk_mass_of_few_queries_over_many_rows(ctx, n, G):
    """Running sums over 70 tiles: what each leaves must not add up.  A score's terms are right to 2^-22 and there are fp32 roundings of
    scores of up to 30 in units of log2 (30 * 2^-24 = 2e-6, ln 2 of it in a weight); sums of 9000 positive terms in 32 chains
    leave sqrt(280) 2^-24 = 1e-6: 4e-6 in all."""
    T = 9000
    k, _ = caches(1, 1, 2, T, torch.bfloat16, 26 + n)
    q = queries((1, 2 * G, n, 128), torch.bfloat16, 4)
    mass = torch.zeros(1, 1, 2, T, device="cuda")
    ctx.attend_mass(k, 0, q, mass, [T])
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       torch.arange(T, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(64, device="cuda").double() / 64))
    z = lambda x, at: torch.complex(x[..., :64].double(), x[..., 64:].double()) * at
    hidden = torch.full((n, T), -torch.inf, dtype=torch.float64, device="cuda").triu(T - n + 1)
    for h in range(2):
        s = (z(q[0, G * h:G * h + G], turn[T - n:]) @ z(k[0, 0, h], turn).conj().T).real / 128 ** 0.5 + hidden
        want = torch.softmax(s, -1).sum((0, 1))
        assert float((mass[0, 0, h].double() - want).norm() / want.norm()) <= 4e-6


def test_chunk_mass_captured_and_refused(ctx):
    k, _ = caches(1, 2, 2, 300, torch.bfloat16, 25)
    q, mass = queries((1, 4, 70, 128), torch.bfloat16, 4), torch.zeros(1, 2, 2, 300, device="cuda")
    ctx.attend_mass(k, 1, q, mass, [222])
    once = mass.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.attend_mass(k, 1, q, mass, [222])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(mass, 2 * once)
    for kw in ({"lens": [69]}, {"lens": [301]}, {"layer": 2}, {"scale": float("nan")}, {"mass": mass[..., :32]}, {"q": q.float()}, {"k": k.float()}):
        a = dict(k=k, layer=0, q=q, mass=mass, lens=[222]) | kw
        with pytest.raises(fk.FreqKVError):
            ctx.attend_mass(**a)
    assert torch.equal(mass, 2 * once)


def test_weights_back_to_back_on_streams_in_turn(ctx):
    """Layer after layer without a wait, streams in turn, decode and chunk calls that share the context's work areas: the sums of the calls
    alone, bit for bit."""
    k, v = caches(2, 3, 2, 1500, torch.bfloat16, 31)
    one, chunk = queries((2, 8, 128), torch.bfloat16, 5), queries((2, 8, 150, 128), torch.bfloat16, 6)
    lens = [1500, 160]
    want = torch.zeros(2, 3, 2, 1500, device="cuda")
    for layer in range(3):
        ctx.attend_decode_mass(k, v, layer, one, want, lens)
        torch.cuda.synchronize()
        ctx.attend_mass(k, layer, chunk, want, lens)
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = torch.zeros_like(want)
    torch.cuda.synchronize()
    for layer in range(3):
        with torch.cuda.stream(streams[layer % 2]):
            ctx.attend_decode_mass(k, v, layer, one, got, lens)
        with torch.cuda.stream(streams[(layer + 1) % 2]):
            ctx.attend_mass(k, layer, chunk, got, lens)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert ctx.last_device_status() == fk.OK


# ---- eviction ----

def check_evict(ctx, k, v, mass, lens, kept, sink, recent, in_place=True, with_rows=True):
    B, L, H, cap, _ = k.shape
    k0, v0, m0 = k.clone(), v.clone(), mass.clone()
    out = mass if in_place else torch.full_like(mass, 3.25)
    o0 = out.clone()
    rows = torch.full((B, L, H, cap), -7, dtype=torch.int32, device="cuda") if with_rows else None
    assert ctx.evict(k, v, mass, lens, kept, sink, recent, mass_out=None if in_place else out, kept_rows=rows) == [sink + x for x in kept]
    if not in_place:
        assert torch.equal(mass.view(torch.int32), m0.view(torch.int32))
    m_host = m0.double().cpu().numpy()
    for b, l, h in np.ndindex(B, L, H):
        stay = oe.keep(m_host[b, l, h], lens[b], kept[b], sink, recent)
        n, idx = len(stay), torch.tensor(stay, dtype=torch.long, device="cuda")
        assert n == sink + kept[b]
        if with_rows:
            assert rows[b, l, h, :n].tolist() == stay and bool((rows[b, l, h, n:] == -7).all())
        as_bits = (torch.int16 if k.dtype == torch.bfloat16 else torch.int32)
        for x, x0 in ((k, k0), (v, v0)):
            got, had = x[b, l, h].view(as_bits), x0[b, l, h].view(as_bits)
            assert torch.equal(got[:n], had[idx]) and torch.equal(got[n:], had[n:])
        got, had, was = (t[b, l, h].view(torch.int32) for t in (out, m0, o0))
        assert torch.equal(got[:n], had[idx]) and not bool(got[n:lens[b]].any()) and torch.equal(got[lens[b]:], was[lens[b]:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cap,lens,kept,sink,recent", [
    (300, [300, 100, 17], [148, 50, 13], 4, 8), (64, [64, 1, 0], [64, 1, 0], 0, 0), (64, [64, 30, 5], [0, 0, 0], 5, 0),
    (700, [700, 513, 512], [10, 512, 300], 0, 10), (1500, [1500, 1025, 600], [1, 1024, 1], 1, 0), (130, [130, 129, 128], [100, 101, 102], 2, 100)])
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(ctx, dtype, cap, lens, kept, sink, recent, in_place):
    k, v = caches(3, 2, 2, cap, dtype, cap)
    check_evict(ctx, k, v, masses((3, 2, 2, cap), cap), lens, kept, sink, recent, in_place, with_rows=cap != 300)


@pytest.mark.parametrize("hd", [8, 24, 64, 80, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_evict_head_sizes_strides_and_slices(ctx, hd, dtype):
    """Padded rows and swapped axes; few matrices, so that their rows go in slices; guard values around them stay."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(hd)
    full = [torch.randn(2, 400, 3, 1, hd + 8, generator=gen, device="cuda").to(dtype) for _ in range(2)]
    before = [f[..., hd:].clone() for f in full]
    k, v = (f.permute(0, 3, 2, 1, 4)[..., :hd] for f in full)     # [batch, layers, heads, tokens, channels]
    check_evict(ctx, k, v, masses((2, 1, 3, 400), hd), [400, 333], [200, 123], 4, 16)
    for f, x in zip(full, before):
        assert torch.equal(f[..., hd:], x)


def test_evict_ties_zeros_nan_and_infinities(ctx):
    cap = 640
    k, v = caches(1, 1, 6, cap, torch.bfloat16, 3)
    mass = torch.zeros(1, 1, 6, cap, device="cuda")
    mass[0, 0, 0] = 0.5                                            # all equal
    mass[0, 0, 1, ::3] = -0.0
    mass[0, 0, 2] = torch.arange(cap, device="cuda") % 7           # many ties at every border
    mass[0, 0, 3] = masses((cap,), 5)
    mass[0, 0, 3, 10:40:3] = float("nan")
    mass[0, 0, 3, 100:140] = float("inf")
    mass[0, 0, 3, 200:240] = -float("inf")
    mass[0, 0, 4] = -masses((cap,), 6)
    mass[0, 0, 5] = 1.0 + 2.0 ** -23 * (torch.arange(cap, device="cuda") * 37 % 5)   # apart in the last bit
    for kept in (20, 63, 64, 300, 500, 620):
        kk, vv, mm = k.clone(), v.clone(), mass.clone()
        check_evict(ctx, kk, vv, mm, [cap], [kept], 3, 10, in_place=False)


def test_evict_many_sequences_long_rows_and_capture(ctx):
    B = 131
    k, v = caches(B, 1, 1, 60, torch.bfloat16, 4)
    lens = [10 + (13 * b) % 50 for b in range(B)]
    check_evict(ctx, k, v, masses((B, 1, 1, 60), 8), lens, [(n - 2) // 2 for n in lens], 2, 3)
    k, v = caches(1, 1, 1, 40000, torch.bfloat16, 5)               # one matrix pair, many rows
    check_evict(ctx, k, v, masses((1, 1, 1, 40000), 9), [39999], [20001], 4, 100)
    k, v = caches(2, 1, 2, 500, torch.bfloat16, 6)
    mass, rows = masses((2, 1, 2, 500), 10), torch.zeros(2, 1, 2, 500, dtype=torch.int32, device="cuda")
    k1, v1, m1 = k.clone(), v.clone(), mass.clone()
    ctx.evict(k1, v1, m1, [500, 400], [200, 100], 4, 10)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.evict(k, v, mass, [500, 400], [200, 100], 4, 10, kept_rows=rows)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(k, k1) and torch.equal(v, v1) and torch.equal(mass, m1)


def test_evict_past_32_bits(ctx):
    """Matrices of one cache more than 4 GB apart."""
    cap, hd = 9_000_000, 256
    k, v = (torch.zeros(1, 1, 2, cap, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n = 3000
    for x in (k, v):
        x[:, :, :, :n] = queries((1, 1, 2, n, hd), torch.bfloat16, 3)
    mass = torch.zeros(1, 1, 2, cap, device="cuda")
    mass[..., :n] = masses((1, 1, 2, n), 4)
    was, m = k[..., :n, :].clone(), mass[..., :n].double().cpu().numpy()
    assert ctx.evict(k, v, mass, [n], [1000], 4, 50) == [1004]
    for h in range(2):
        idx = torch.tensor(oe.keep(m[0, 0, h], n, 1000, 4, 50), device="cuda")
        assert torch.equal(k[0, 0, h, :1004], was[0, 0, h][idx]) and torch.equal(v[0, 0, h, :1004], was[0, 0, h][idx])
    assert not bool(k[0, 0, :, n:n + 1000].any())


def test_evict_refusals(ctx):
    k, v = caches(1, 2, 2, 64, torch.bfloat16, 17)
    mass = masses((1, 2, 2, 64), 3)
    k0, m0 = k.clone(), mass.clone()
    for kw in ({"lens": [65]}, {"kept_len": [61]}, {"kept_len": [7]}, {"sink": -1}, {"recent": -1}, {"mass": mass.half()}, {"kept_rows": mass},
               {"mass_out": mass[:, :1]}, {"lens": [3]}, {"lens": [64, 64]}):
        a = dict(k=k, v=v, mass=mass, lens=[64], kept_len=[30], sink=4, recent=8) | kw
        with pytest.raises(fk.FreqKVError):
            ctx.evict(**a)
    assert torch.equal(k, k0) and torch.equal(mass, m0)


def test_a_stream_with_eviction(ctx):
    """As they are used: a prompt in chunks, then tokens, weights added up all the way, the full cache evicted twice: the rows that
    stay are the oracle's choice by the masses, and every query has given away a weight of one."""
    B, L, H, cap, G, sink, recent = 2, 2, 2, 256, 4, 4, 32
    k, v = (torch.zeros(B, L, H, cap, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mass, lens, seed = torch.zeros(B, L, H, cap, device="cuda"), [0] * B, 70
    for n in (128, 128, None, 100, 1, 1, 24, None, 1, 1):
        seed += 1
        if n is None:
            with pytest.raises(fk.FreqKVError) as e:
                ctx.append(k, v, new[0][:, :, :, :1].contiguous(), new[1][:, :, :, :1].contiguous(), lens)
            assert e.value.status == fk.ERR_CAPACITY
            assert abs(float(mass.double().sum()) - seen) <= 1e-4 * seen
            k0, v0, m0, had = k.clone(), v.clone(), mass.clone(), lens
            kept = [(x - sink) // 2 for x in lens]
            lens = ctx.evict(k, v, mass, lens, kept, sink, recent)
            m_host = m0.double().cpu().numpy()
            for b, l, h in np.ndindex(B, L, H):
                idx = torch.tensor(oe.keep(m_host[b, l, h], had[b], kept[b], sink, recent), device="cuda")
                assert torch.equal(k[b, l, h, :lens[b]], k0[b, l, h][idx]) and torch.equal(v[b, l, h, :lens[b]], v0[b, l, h][idx])
                assert torch.equal(mass[b, l, h, :lens[b]], m0[b, l, h][idx]) and not bool(mass[b, l, h, lens[b]:].any())
            continue
        seen = float(mass.double().sum()) + B * L * H * G * n      # every query gives away one
        new = [queries((B, L, H, n, 128), torch.bfloat16, seed + 100 * i) for i in range(2)]
        lens = ctx.append(k, v, *new, lens)
        for layer in range(L):
            q = queries((B, H * G, n, 128), torch.bfloat16, seed + layer)
            if n == 1:
                one = q[:, :, 0].contiguous()
                a, b = ctx.attend_decode_mass(k, v, layer, one, mass, lens), ctx.attend_decode(k, v, layer, one, lens)
                assert float((a.float() - b.float()).norm() / b.float().norm()) <= 2 * OUT[torch.bfloat16]
            else:
                ctx.attend_prefill(k, v, layer, q, lens)
                ctx.attend_mass(k, layer, q, mass, lens)
        assert abs(float(mass.double().sum()) - seen) <= 1e-4 * seen
    assert ctx.last_device_status() == fk.OK
