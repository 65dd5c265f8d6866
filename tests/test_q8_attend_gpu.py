"""Attention over the 8-bit cache against the 64-bit oracle on the values that the codes stand for.

Tolerance, relative L2 of one query head's 128 channels.  The result is rounded to bf16: at most 2^-8.  Scores: a turned key channel
carries the roundings of a cosine, two products and a sum, a query channel one, each at most 2^-11 of a term, independent over
128 channels: a score of standard deviation sigma is off by about sqrt(5) 2^-11 sigma / sqrt(3) (a rounding's root mean
square is its most over sqrt(3)), and the weighted mean of values by that share of itself where the values are independent: with
sigma up to 8 (these inputs), 5e-3 -- in the worst case of weights that all sit on two rows of opposite values, twice that.
Weights: 2^-11.  Sum: 4e-3 + 1e-2 + 1e-3, tolerance 1.5e-2; the matrix of all heads together has to keep 5e-3."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2505_00570_b200 import binding as fk
from tests.test_q8_gpu import rows

pytestmark = pytest.mark.gpu

KIND = {"int8": fk.Q8_INT8, "e4m3": fk.Q8_E4M3}
ONE_HEAD, ALL = 1.5e-2, 5e-3


@pytest.fixture(scope="module")
def ctx():
    c = fk.Context(0)
    yield c
    c.close()


def make(ctx, B, L, H, cap, kind, block, seed=1, spread=0.5, row_pad=0):
    """A full cache of rows of different sizes, two loud channels a head, and the values that it stands for in 64 bits."""
    dtype = torch.int8 if kind == "int8" else torch.float8_e4m3fn
    codes = [torch.zeros(B, L, H, cap, 128 + row_pad, dtype=torch.int8, device="cuda").view(dtype)[..., :128] for _ in range(2)]
    scales = [torch.zeros(B, L, H, -(-cap // block), device="cuda") for _ in range(2)]
    cache = fk.Q8Cache(*codes, *scales, block)
    k, v = (rows((B, L, H, cap, 128), torch.bfloat16, 31 * seed + i, spread) for i in range(2))
    k[..., 5] *= 4
    k[..., 77] *= 4
    ctx.quantize(k, v, [cap] * B, cache)
    return cache


def values(cache):
    return [(c.to(torch.float32).double() * s.double().repeat_interleave(cache.block_tokens, 3)[..., :c.shape[3], None]).cpu().numpy()
            for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]


def queries(shape, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)


def near(got, want):
    got, want = got.double().cpu().numpy().reshape(-1, 128), np.asarray(want).reshape(-1, 128)
    assert np.isfinite(got).all()
    off = np.linalg.norm(got - want, axis=1) / np.linalg.norm(want, axis=1)
    assert off.max() <= ONE_HEAD, (off.argmax(), off.max())
    whole = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert whole <= ALL, whole


def check_decode(ctx, cache, layer, q, lens, base=10000.0, scale=0.0, kv=None, heads=None):
    out = ctx.attend_decode_q8(cache, layer, q, lens, rope_base=base, scale=scale)
    assert ctx.last_device_status() == fk.OK
    k, v = kv if kv is not None else values(cache)
    G = q.shape[1] // k.shape[2]
    picked = heads or [(b, h) for b in range(q.shape[0]) for h in range(k.shape[2])]
    want = [oa.attend_decode(q[b, h * G:(h + 1) * G].double().cpu().numpy(), k[b, layer, h], v[b, layer, h], lens[b], base,
                             None if scale <= 0 else scale) for b, h in picked]
    near(torch.stack([out[b, h * G:(h + 1) * G] for b, h in picked]), np.stack(want))
    return out


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 9, 16, 21])
def test_decode_head_groups(ctx, kind, G):
    cache = make(ctx, 3, 2, 2, 300, kind, 32, seed=G)
    before = [x.clone() for x in (cache.k.view(torch.int8), cache.v.view(torch.int8), cache.k_scale, cache.v_scale)]
    check_decode(ctx, cache, 1, queries((3, 2 * G, 128), 5 + G), [300, 37, 1])
    for x, y in zip((cache.k.view(torch.int8), cache.v.view(torch.int8), cache.k_scale, cache.v_scale), before):
        assert torch.equal(x, y)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_decode_lengths_around_tiles_blocks_and_splits(ctx, kind, block):
    cache = make(ctx, 1, 1, 2, 1100, kind, block, seed=block, row_pad=16)
    kv = values(cache)
    q = queries((1, 8, 128), 6)
    for n in (1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 1023, 1024, 1025, 1099, 1100):
        check_decode(ctx, cache, 0, q, [n], kv=kv)


@pytest.mark.parametrize("base,scale", [(0.0, 0.0), (500000.0, 0.05), (10000.0, 0.2)])
def test_decode_rope_off_other_base_and_scale(ctx, base, scale):
    cache = make(ctx, 2, 2, 3, 200, "e4m3", 64, seed=12, spread=0.3)
    check_decode(ctx, cache, 0, queries((2, 6, 128), 3), [199, 64], base, scale)
    check_decode(ctx, cache, 1, queries((2, 6, 128), 4), [2, 200], base, scale)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_decode_small_capacity(ctx, kind):
    """Fewer rows than the table of the tile's angles has."""
    cache = make(ctx, 2, 1, 1, 3, kind, 16, seed=3)
    c = fk.Context(0)
    check_decode(c, cache, 0, queries((2, 2, 128), 3), [3, 1])
    c.close()


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_decode_scales_of_any_size(ctx, kind):
    """V's scales from 2^-100 to 2^100 in one sequence, blocks of zeros among them; rows behind the last full of NaN."""
    cache = make(ctx, 1, 1, 2, 640, kind, 64, seed=8)
    for i, e in enumerate((-100, -3, 0, None, 5, 40, 39, 100, None, 98)):
        block = cache.v_scale[0, 0, :, i]
        block.mul_(0.0 if e is None else 2.0 ** e)
    kv = values(cache)
    if kind == "e4m3":
        for c in (cache.k, cache.v):
            c.view(torch.int8)[:, :, :, 630:] = 0x7f
    q = queries((1, 4, 128), 9)
    for n in (30, 128, 200, 256, 320, 630):
        out = ctx.attend_decode_q8(cache, 0, q, [n])
        want = np.concatenate([oa.attend_decode(q[0, 2 * h:2 * h + 2].double().cpu().numpy(), kv[0][0, 0, h], kv[1][0, 0, h], n, 10000.0) for h in range(2)])
        near(out, want)


def test_decode_codes_that_are_nan_stay_in_their_channel_or_row(ctx):
    cache = make(ctx, 1, 1, 2, 100, "e4m3", 16, seed=9)
    q = queries((1, 2, 128), 9)
    clean = ctx.attend_decode_q8(cache, 0, q, [100])
    cache.v.view(torch.int8)[0, 0, 0, 50, 3] = 0x7f
    out = ctx.attend_decode_q8(cache, 0, q, [100])
    assert bool(out[0, 0, 3].isnan()) and int(out.isnan().sum()) == 1
    keep = ~out.isnan()
    assert torch.equal(out[keep], clean[keep])
    assert torch.equal(ctx.attend_decode_q8(cache, 0, q, [50])[0, 1], ctx.attend_decode_q8(cache, 0, q, [50])[0, 1])
    cache.k.view(torch.int8)[0, 0, 1, 7, 3] = 0x7f
    out = ctx.attend_decode_q8(cache, 0, q, [100])
    assert bool(out[0, 1].isnan().all()) and not bool(out[0, 0, 4:].isnan().any())


def test_decode_one_key_wins_and_uniform_keys(ctx):
    cache = fk.Q8Cache.empty(1, 1, 1, 128, 128, fk.Q8_INT8, 16)
    k = torch.zeros(1, 1, 1, 128, 128, device="cuda", dtype=torch.bfloat16)
    v = torch.randn(1, 1, 1, 128, 128, device="cuda").to(torch.bfloat16)
    q = torch.zeros(1, 1, 128, device="cuda", dtype=torch.bfloat16)
    q[0, 0, 0] = 1.0
    ctx.quantize(k, v, [128], cache)
    vv = torch.from_numpy(values(cache)[1])[0, 0, 0]
    out = ctx.attend_decode_q8(cache, 0, q, [100], rope_base=0.0)
    assert torch.allclose(out[0, 0].double().cpu(), vv[:100].mean(0), atol=2 ** -8 * float(vv[:100].mean(0).abs().max()) + 1e-3)
    k[0, 0, 0, 41, 0] = 2000.0
    ctx.quantize(k, v, [128], cache)
    out = ctx.attend_decode_q8(cache, 0, q, [100], rope_base=0.0)
    assert torch.allclose(out[0, 0].double().cpu(), vv[41], rtol=2 ** -8, atol=1e-4)


def test_decode_many_sequences_and_captured(ctx):
    """More sequences than one launch takes; then the same call captured and replayed, its queries changed in between."""
    B = 130
    cache = make(ctx, B, 1, 1, 80, "e4m3", 16, seed=13)
    lens = [1 + (37 * b) % 80 for b in range(B)]
    q = queries((B, 2, 128), 3)
    kv = values(cache)
    out = check_decode(ctx, cache, 0, q, lens, kv=kv)
    long = make(ctx, 1, 1, 1, 3000, "int8", 32, seed=14)
    ql, got = queries((1, 3, 128), 4), torch.empty(1, 3, 128, dtype=torch.bfloat16, device="cuda")
    first = ctx.attend_decode_q8(long, 0, ql, [3000]).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.attend_decode_q8(long, 0, ql, [3000], out=got, stream=torch.cuda.current_stream())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.allclose(got.float(), first.float(), rtol=2 ** -7, atol=1e-3)
    ql.copy_(queries((1, 3, 128), 5))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.allclose(got.float(), ctx.attend_decode_q8(long, 0, ql, [3000]).float(), rtol=2 ** -7, atol=1e-3)
    assert torch.equal(ctx.attend_decode_q8(cache, 0, q, lens), out)   # the same call gives the same bits


def test_decode_ragged_lengths_in_many_splits_back_to_back(ctx):
    """Sequences of one row beside long ones, layer after layer without a wait, bases in turn (each makes its table anew), other calls of
    the context between them: every result is that of the call alone."""
    cache = make(ctx, 3, 3, 2, 4000, "e4m3", 32, seed=15)
    k, v = rows((3, 1, 2, 500, 128), torch.bfloat16, 3), rows((3, 1, 2, 500, 128), torch.bfloat16, 4)
    q, lens = queries((3, 8, 128), 3), [1, 4000, 17]
    alone = {}
    for layer in range(3):
        for base in (10000.0, 500000.0):
            alone[layer, base] = ctx.attend_decode_q8(cache, layer, q, lens, rope_base=base).clone()
            torch.cuda.synchronize()
    kv = values(cache)
    for layer in (0, 2):
        check_decode(ctx, cache, layer, q, lens, kv=kv)
    got = []
    for _ in range(3):
        for base in (10000.0, 500000.0):
            for layer in range(3):
                got.append((layer, base, ctx.attend_decode_q8(cache, layer, q, lens, rope_base=base)))
            ctx.attend_decode(k, v, 0, q, [500, 3, 70], rope_base=base)
    for layer, base, out in got:
        assert torch.equal(out, alone[layer, base])


def test_two_contexts_on_two_streams(ctx):
    other = fk.Context(0)
    a, b = make(ctx, 2, 1, 4, 3000, "e4m3", 64, seed=16), make(ctx, 2, 1, 4, 3000, "int8", 16, seed=17)
    qa, qb = queries((2, 16, 128), 3), queries((2, 4, 128), 4)
    chunk = queries((2, 16, 200, 128), 5)
    want = [ctx.attend_decode_q8(a, 0, qa, [3000, 2000]), ctx.attend_decode_q8(b, 0, qb, [700, 3000]), ctx.attend_prefill_q8(a, 0, chunk, [3000, 777])]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            x, z = ctx.attend_decode_q8(a, 0, qa, [3000, 2000]), ctx.attend_prefill_q8(a, 0, chunk, [3000, 777])
        with torch.cuda.stream(streams[1]):
            y = other.attend_decode_q8(b, 0, qb, [700, 3000])
        got.append((x, y, z))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(p, w) for p, w in zip(g, want))
    # one context, streams in turn: its calls follow one another
    outs = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(ctx.attend_decode_q8(a, 0, qa, [3000, 2000]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) for o in outs)
    other.close()


def test_decode_long_cache_and_offsets_past_32_bits(ctx):
    cap = 9_000_000                                    # 128 bytes a row: one matrix past 1 GB, the second head past 2^30 rows' bytes
    cache = fk.Q8Cache.empty(1, 2, 2, cap, 128, fk.Q8_INT8, 128)
    n = 5000
    new = [rows((1, 2, 2, n, 128), torch.bfloat16, 60 + i, 0.3) for i in range(2)]
    ctx.append_q8(cache, *new, [0])
    q = queries((1, 8, 128), 3)
    small = fk.Q8Cache(*[c[..., :n + 24, :] for c in (cache.k, cache.v)],
                       *[s[..., :(n + 24 + 127) // 128].contiguous() for s in (cache.k_scale, cache.v_scale)], 128)
    kv = values(small)
    out = ctx.attend_decode_q8(small, 1, q, [n])
    want = np.concatenate([oa.attend_decode(q[0, 4 * h:4 * h + 4].double().cpu().numpy(), kv[0][0, 1, h], kv[1][0, 1, h], n, 10000.0) for h in range(2)])
    near(out, want)


def test_decode_refusals(ctx):
    cache = make(ctx, 1, 2, 2, 64, "int8", 32)
    q = queries((1, 2, 128), 3)
    for bad in ([0], [65]):
        with pytest.raises(fk.FreqKVError) as e:
            ctx.attend_decode_q8(cache, 0, q, bad)
        assert e.value.status == fk.ERR_INVALID_ARG
    for kw in ({"scale": float("nan")}, {"rope_base": float("nan")}):
        with pytest.raises(fk.FreqKVError):
            ctx.attend_decode_q8(cache, 0, q, [5], **kw)
    with pytest.raises(fk.FreqKVError):
        ctx.attend_decode_q8(cache, 2, q, [5])
    with pytest.raises(fk.FreqKVError):
        ctx.attend_decode_q8(cache, 0, q, [5], out=q)
    with pytest.raises(fk.FreqKVError):
        ctx.attend_decode_q8(cache, 0, q.float(), [5])
    with pytest.raises(fk.FreqKVError) as e:
        ctx.attend_decode_q8(cache, 0, queries((1, 130, 128), 3), [5])
    assert e.value.status == fk.ERR_UNSUPPORTED


# ---- chunks ----

def check_prefill(ctx, cache, layer, q, lens, base=10000.0, scale=0.0, kv=None, heads=None):
    out = ctx.attend_prefill_q8(cache, layer, q, lens, rope_base=base, scale=scale)
    assert ctx.last_device_status() == fk.OK
    k, v = kv if kv is not None else values(cache)
    B, Hq, n, _ = q.shape
    G = Hq // k.shape[2]
    for b, h in heads or [(b, h) for b in range(B) for h in range(Hq)]:
        tokens = sorted({0, 1, n // 2, n - 1} | {t for t in (63, 64, 127, 128, 129) if t < n})
        want = [oa.attend_decode(q[b, h:h + 1, t].double().cpu().numpy(), k[b, layer, h // G], v[b, layer, h // G], lens[b] - n + t + 1, base,
                                 None if scale <= 0 else scale) for t in tokens if t < n]
        near(out[b, h, [t for t in tokens if t < n]], np.stack(want))
    return out


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("G,n,lens,block", [(1, 1, [1, 70], 16), (2, 2, [2, 3], 32), (3, 64, [64, 200], 64), (4, 129, [129, 300], 128),
                                            (1, 200, [230, 299], 16), (9, 5, [65, 128], 64)])
def test_prefill_small(ctx, kind, G, n, lens, block):
    cache = make(ctx, 2, 2, 2, 300, kind, block, seed=n, row_pad=16)
    check_prefill(ctx, cache, 1, queries((2, 2 * G, n, 128), n), lens)


@pytest.mark.parametrize("base,scale", [(0.0, 0.0), (500000.0, 0.05)])
def test_prefill_rope_off_other_base_and_scale(ctx, base, scale):
    cache = make(ctx, 1, 1, 2, 500, "e4m3", 64, seed=21, spread=0.3)
    check_prefill(ctx, cache, 0, queries((1, 4, 130, 128), 3), [497], base, scale)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_prefill_scales_of_any_size_and_rows_behind_the_last(ctx, kind):
    cache = make(ctx, 1, 1, 1, 640, kind, 64, seed=22)
    for i, e in enumerate((60, 58, 59, None, 60, 57, 60, 55, 60, 60)):
        cache.v_scale[0, 0, :, i].mul_(0.0 if e is None else 2.0 ** e)
    kv = values(cache)
    if kind == "e4m3":
        for c in (cache.k, cache.v):
            c.view(torch.int8)[:, :, :, 570:] = 0x7f
    check_prefill(ctx, cache, 0, queries((1, 2, 300, 128), 3), [570], kv=kv)


def test_prefill_of_one_token_is_decoding(ctx):
    cache = make(ctx, 2, 1, 2, 777, "int8", 32, seed=23)
    q = queries((2, 8, 128), 4)
    a, b = ctx.attend_decode_q8(cache, 0, q, [777, 5]), ctx.attend_prefill_q8(cache, 0, q.unsqueeze(2), [777, 5])
    assert float((a.float() - b.squeeze(2).float()).norm() / a.float().norm()) <= 2 * ALL


def test_a_stream_in_8_bits(ctx):
    """As they are used: chunks are appended and attend, the full cache goes out, is compressed and comes back, tokens are appended
    and attend.  The attention is compared with the bf16 calls on the same rows, dequantized."""
    B, L, H, cap, G, sink = 2, 2, 2, 320, 4, 4
    cache = fk.Q8Cache.empty(B, L, H, cap, kind=fk.Q8_E4M3, block_tokens=32)
    work = [torch.zeros(B, L, H, cap, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens, seed = [0, 0], 40
    for n in (160, 160, None, 100, 1, 1, 56):
        seed += 1
        if n is None:                                  # full: e4m3 values are exact in bf16
            with pytest.raises(fk.FreqKVError) as e:
                ctx.append_q8(cache, new[0][:, :, :, :1].contiguous(), new[1][:, :, :, :1].contiguous(), lens)
            assert e.value.status == fk.ERR_CAPACITY
            ctx.dequantize(cache, lens, *work)
            kept = (cap - sink) // 2
            lens = [ctx.compress(*work, cap, kept, sink)] * B
            ctx.quantize(*work, lens, cache)
            continue
        new = [rows((B, L, H, n, 128), torch.bfloat16, seed + 100 * i, 0.3) for i in range(2)]
        lens = ctx.append_q8(cache, *new, lens)
        ctx.dequantize(cache, lens, *work)
        for layer in range(L):
            q = queries((B, H * G, n, 128), seed + layer)
            if n == 1:
                a, b = ctx.attend_decode_q8(cache, layer, q[:, :, 0].contiguous(), lens), ctx.attend_decode(*work, layer, q[:, :, 0].contiguous(), lens)
            else:
                a, b = ctx.attend_prefill_q8(cache, layer, q, lens), ctx.attend_prefill(*work, layer, q, lens)
            assert float((a.float() - b.float()).norm() / b.float().norm()) <= 2 * ALL
    assert ctx.last_device_status() == fk.OK
    assert lens == [sink + 158 + 158] * B
