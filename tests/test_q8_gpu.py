"""Rows into the 8-bit cache and out of it, against the 64-bit statement of oracle/q8.py.

Scales and codes have one right value each, so both are compared bit for bit; so are the values that come out (code * scale is exact in
64 bits and rounded once)."""
import numpy as np
import pytest
import torch

from oracle import q8
from paper_2505_00570_b200 import binding as fk

pytestmark = pytest.mark.gpu

KINDS = {"int8": fk.Q8_INT8, "e4m3": fk.Q8_E4M3}


@pytest.fixture(scope="module")
def ctx():
    c = fk.Context(0)
    yield c
    c.close()


def rows(shape, dtype, seed, spread=2.0):
    """Rows of very different magnitudes, so that appended ones outgrow the scales of their blocks."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * (torch.randn(shape[:-1], generator=gen, device="cuda") * spread).exp()[..., None]).to(dtype).contiguous()


def cache_of(B, L, H, cap, hd, kind, block, seed=1, row_pad=0):
    """A cache whose every byte is set, in padded rows where asked: nothing outside the written rows may change."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = torch.int8 if kind == "int8" else torch.float8_e4m3fn
    codes = [torch.randint(-100, 100, (B, L, H, cap, hd + row_pad), generator=gen, device="cuda", dtype=torch.int8).view(dtype)[..., :hd]
             for _ in range(2)]
    scales = [torch.rand(B, L, H, -(-cap // block), generator=gen, device="cuda") for _ in range(2)]
    if kind == "e4m3":
        scales = [torch.exp2(torch.floor(torch.log2(s))) for s in scales]
    return fk.Q8Cache(*codes, *scales, block)


def state(cache):
    return [c.to(torch.float32).double().cpu().numpy() for c in (cache.k, cache.v)], [s.double().cpu().numpy() for s in (cache.k_scale, cache.v_scale)]


def expect(before, new, begin, n, kind, block):
    """The state after rows enter behind begin[b] (n[b] of them), all matrices."""
    codes, scales = [[np.array(x) for x in part] for part in before]
    for i in range(2):
        src = new[i].double().cpu().numpy()
        for b, l, h in np.ndindex(codes[i].shape[:3]):
            codes[i][b, l, h], scales[i][b, l, h] = q8.append(codes[i][b, l, h], scales[i][b, l, h], src[b, l, h, :n[b]], begin[b], kind, block)
    return codes, scales


def same(cache, want):
    got = state(cache)
    for g, w in zip(got[0] + got[1], want[0] + want[1]):
        assert np.array_equal(g, w, equal_nan=True), np.argwhere(~((g == w) | (np.isnan(g) & np.isnan(w))))[:5]


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_rows_at_every_place_of_a_block(ctx, kind, block, dtype):
    cap = 300
    cache = cache_of(3, 2, 2, cap, 128, kind, block, row_pad=16)
    for seed, (lens, n) in enumerate([([0, 1, block - 1], 1), ([block, 17, 255], 1), ([0, 5, min(200, cap - block)], block), ([3, 0, 100], 2 * block + 5 if block < 64 else 150),
                                      ([cap - 1, 0, 31], 1), ([0, 0, 0], cap)]):
        new = [rows((3, 2, 2, n, 128), dtype, 10 * seed + i) for i in range(2)]
        want = expect(state(cache), new, lens, [n] * 3, kind, block)
        assert ctx.append_q8(cache, *new, lens) == [x + n for x in lens]
        same(cache, want)
    assert ctx.append_q8(cache, new[0][:, :, :, :0].contiguous(), new[1][:, :, :, :0].contiguous(), [300, 0, 1]) == [300, 0, 1]
    with pytest.raises(fk.FreqKVError) as e:
        ctx.append_q8(cache, *new, [1, 0, 0])
    assert e.value.status == fk.ERR_CAPACITY


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_append_token_by_token(ctx, kind):
    """The stream of a decode loop: every step may move the scale of the block it is in."""
    cache = cache_of(1, 1, 2, 48, 128, kind, 32)
    lens = [0]
    for t in range(48):
        new = [rows((1, 1, 2, 1, 128), torch.bfloat16, 100 + 2 * t + i) for i in range(2)]
        want = expect(state(cache), new, lens, [1], kind, 32)
        lens = ctx.append_q8(cache, *new, lens)
        same(cache, want)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("hd,block", [(16, 16), (64, 64), (80, 32), (256, 128), (240, 16), (128, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_and_back(ctx, kind, hd, block, dtype):
    lens = [150, 0, 1, 97]
    cache = cache_of(4, 1, 3, 160, hd, kind, block)
    src = [rows((4, 3, 1, 151, hd + 8), dtype, 7 + i).transpose(1, 2)[..., :hd] for i in range(2)]      # padded rows, axes swapped
    want = expect(state(cache), src, [0] * 4, lens, kind, block)
    ctx.quantize(*src, lens, cache)
    same(cache, want)
    for out in (torch.float32, torch.bfloat16):
        back = [torch.full((4, 1, 3, 155, hd), 7.0, dtype=out, device="cuda") for _ in range(2)]
        ctx.dequantize(cache, lens, *back)
        for i in range(2):
            for b, h in np.ndindex(4, 3):
                v = q8.values(want[0][i][b, 0, h], want[1][i][b, 0, h], block)[:lens[b]]
                v = torch.from_numpy(v).to(torch.float32).to(out)
                assert torch.equal(back[i][b, 0, h, :lens[b]].cpu(), v)
                assert bool((back[i][b, 0, h, lens[b]:] == 7.0).all())
    same(cache, want)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_at_the_borders(ctx, kind, dtype):
    """Ties, infinities, NaN, zeros, subnormals and the largest values, each in a block of its own."""
    block, hd = 16, 128
    src = torch.zeros(1, 1, 1, 16 * 12, hd, dtype=torch.float64)
    t = src.view(12, 16 * hd)
    half = torch.arange(-254, 255, dtype=torch.float64) / 2                      # all halves up to 127: ties under scale 1
    t[0, :len(half)] = half
    t[1, :len(half)] = half * 2.0 ** -20
    t[2, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 3.0])
    t[3, 1] = float("nan")                                                        # nothing finite but zeros
    t[3, 2] = float("inf")
    t[5, :3] = torch.tensor([2.0 ** -133, -2.0 ** -130, 2.0 ** -126])              # subnormal scales do not exist
    t[6, :3] = torch.tensor([3.38e38, -3.38e38, 1e30])
    t[7, :3] = torch.tensor([2.0 ** -133, 0.0, -0.0])
    x = torch.arange(0, 16 * hd, dtype=torch.float64) / 3
    t[8] = x
    t[9] = -x * 1.0000001
    t[10, :200] = torch.arange(1, 201, dtype=torch.float64) * 2.0 ** -10            # e4m3 codes that are subnormal
    t[10, 200] = 448.0
    t[11] = torch.linspace(-1, 1, 16 * hd, dtype=torch.float64)
    src = src.to(dtype).cuda()
    cache = cache_of(1, 1, 1, 16 * 12, hd, kind, block)
    want = expect(state(cache), [src, src], [0], [16 * 12], kind, block)
    with np.errstate(all="ignore"):
        ctx.quantize(src, src.clone(), [16 * 12], cache)
    same(cache, want)
    # old codes under a scale that grows by a factor that is no power of two, ties among them
    new = [torch.full((1, 1, 1, 4, hd), v, dtype=dtype, device="cuda") for v in (2 * 127.0, 1e4)]
    want = expect(state(cache), new, [12], [4], kind, block)
    ctx.append_q8(cache, *new, [12])
    same(cache, want)


def test_many_sequences_and_other_streams(ctx):
    """More sequences than one launch takes, on a stream of the caller's."""
    B = 131
    cache = cache_of(B, 1, 1, 40, 64, "e4m3", 16)
    lens = [(7 * b) % 37 for b in range(B)]
    new = [rows((B, 1, 1, 3, 64), torch.bfloat16, 50 + i) for i in range(2)]
    want = expect(state(cache), new, lens, [3] * B, "e4m3", 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ctx.append_q8(cache, *new, lens, stream=side)
    side.synchronize()
    same(cache, want)


def test_offsets_past_32_bits(ctx):
    """One matrix of a cache whose codes span more than 4 GB: the last rows are written and read where they belong."""
    cap, hd, block = 17_000_000, 256, 128
    cache = fk.Q8Cache.empty(1, 1, 1, cap, hd, fk.Q8_INT8, block)
    new = [rows((1, 1, 1, 40, hd), torch.bfloat16, 60 + i) for i in range(2)]
    at = cap - 40
    assert ctx.append_q8(cache, *new, [at]) == [cap]
    first = at // block * block
    for i, (codes, scales) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        want, s = q8.append(np.zeros((cap - first, hd)), np.zeros(-(-(cap - first) // block)), new[i][0, 0, 0].double().cpu().numpy(), at - first,
                            "int8", block)
        assert np.array_equal(codes[0, 0, 0, first:].double().cpu().numpy(), want)
        assert np.array_equal(scales[0, 0, 0, first // block:].double().cpu().numpy(), s)
        assert not bool(codes[0, 0, 0, :first].view(torch.int64).any())


def test_capture_and_replay(ctx):
    """The calls keep no work area: a captured append runs again on what its tensors then hold."""
    cache = cache_of(2, 1, 2, 64, 128, "int8", 32)
    new = [rows((2, 1, 2, 2, 128), torch.bfloat16, 80 + i) for i in range(2)]
    lens = [5, 30]
    before = state(cache)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.append_q8(cache, *new, lens, stream=torch.cuda.current_stream())
    same(cache, before)
    for i in range(2):
        new[i].copy_(rows((2, 1, 2, 2, 128), torch.bfloat16, 90 + i))
    want = expect(state(cache), new, lens, [2, 2], "int8", 32)
    graph.replay()
    torch.cuda.synchronize()
    same(cache, want)
