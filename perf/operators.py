"""The operators of a bounded cache in 8 bits and of eviction by attention weight, as timed cases.

  write    rows enter an 8-bit cache: one token of a decode step, a chunk, or a whole cache (``quantize``);
  decode   one token per sequence attends over the 8-bit cache, layer after layer;
  prefill  a chunk of tokens per sequence attends causally over the 8-bit cache, layer after layer;
  mass     attention weights are added up per cache row: by the decode attention that computes them
           (n_new 1), or by a call of their own for a chunk's queries;
  evict    every cache drops its lightest rows: sinks, recent rows and the heaviest others move together.

``run`` computes the plain form in elementary torch operations, or, where ``own`` is true, calls the library.
Keys and values are moving-average sequences with a few outlier channels, the shape of real key/value states.
"""
from __future__ import annotations

import math

import torch

own = False

SRC = {"bf16": torch.bfloat16, "fp32": torch.float32}
SRC_BYTES = {"bf16": 2, "fp32": 4}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
HEAD = 128
BASE = 10000.0
TINY = 2.0 ** -126


# ---- cases ----------------------------------------------------------------------------------------------------------

def _case(op, batch, layers, kv_heads, capacity, lens, **more):
    return dict(op=op, batch=batch, layers=layers, kv_heads=kv_heads, capacity=capacity, lens=lens, **more)


def listed():
    return [
        # One decode step of a batch of 8: each sequence's new rows enter its last block, for 8 layers of LLaMA-3-8B shapes.
        dict(_case("write", 8, 8, 8, 4096, "4095 3501 3056 2560 4000 2049 3888 3327", how="append", n_new=1, kind="e4m3", block=64,
                   dtype="bf16"), name="q8_append_step"),
        # A whole LLaMA-2-7B cache of 4096 rows goes to 8 bits, as after a compression or a prefill.
        dict(_case("write", 1, 32, 32, 4096, "4096", how="quantize", n_new=4096, kind="int8", block=32, dtype="bf16"), name="q8_quantize_7b"),
        # The smallest attention: one layer of one short sequence.
        dict(_case("decode", 1, 1, 8, 512, "300", group=4, kind="e4m3", block=64), name="q8_decode_small"),
        # A decode step of a batch of 8 on LLaMA-3-8B shapes, long caches of different lengths.
        dict(_case("decode", 8, 8, 8, 8192, "8192 7001 6113 5120 8000 4099 7777 6655", group=4, kind="e4m3", block=64), name="q8_decode_8b"),
        # A decode step of a batch of 16 on LLaMA-2-7B shapes (one query head a KV head), caches full.
        dict(_case("decode", 16, 4, 32, 4096, "4096", group=1, kind="int8", block=32), name="q8_decode_7b"),
        # The chunk that fills a LLaMA-2-7B cache after a compression.
        dict(_case("prefill", 1, 4, 32, 4096, "4096", group=1, n_new=2046, kind="e4m3", block=64), name="q8_prefill_7b"),
        # A short odd chunk for two sequences of LLaMA-3-8B shapes.
        dict(_case("prefill", 2, 4, 8, 8192, "5003 6790", group=4, n_new=1001, kind="int8", block=16), name="q8_prefill_8b_odd"),
        # A decode step that also adds up the weights: a batch of 8 on LLaMA-3-8B shapes.
        dict(_case("mass", 8, 8, 8, 8192, "8192 7001 6113 5120 8000 4099 7777 6655", group=4, n_new=1, dtype="bf16"), name="mass_decode_8b"),
        # The same for a single user.
        dict(_case("mass", 1, 8, 8, 4096, "2611", group=4, n_new=1, dtype="bf16"), name="mass_decode_single"),
        # The weights that a prompt's last chunk gives to the rows.
        dict(_case("mass", 2, 4, 8, 8192, "5003 6790", group=4, n_new=1001, dtype="bf16"), name="mass_chunk_8b_odd"),
        # A full LLaMA-2-7B cache keeps half of its rows.
        dict(_case("evict", 1, 32, 32, 4096, "4096", kept="2046", sink=4, recent=256, dtype="bf16"), name="evict_7b"),
        # One layer of two short sequences of different lengths.
        dict(_case("evict", 2, 1, 8, 2048, "1187 2000", kept="591 998", sink=4, recent=100, dtype="bf16"), name="evict_small"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "decode", "decode", "prefill", "mass", "mass", "evict"])
    kv_heads = rng.choice([1, 4, 8, 8, 32])
    kind, block = rng.choice(["e4m3", "int8"]), rng.choice([16, 32, 64, 128])
    group = 1 if kv_heads == 32 else rng.choice([1, 2, 4, 8])
    capacity = 128 * _log_int(rng, 2, 64)
    low = max(1, capacity // 3)
    if op == "write":
        batch, layers = _log_int(rng, 1, 8), rng.randrange(1, 9)
        how = rng.choice(["append", "append", "quantize"])
        n_new = rng.choice([1, _log_int(rng, 2, capacity // 2)])
        lens = [rng.randrange(0, capacity - n_new + 1) if how == "append" else rng.randrange(low, capacity + 1) for _ in range(batch)]
        return _case("write", batch, layers, min(kv_heads, 8), capacity, " ".join(map(str, lens)), how=how,
                     n_new=n_new if how == "append" else capacity, kind=kind, block=block, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if op == "decode":
        batch = _log_int(rng, 1, 16 if kv_heads <= 8 else 8)
        layers = rng.randrange(1, 9 if kv_heads * batch <= 64 else 5)
        lens = [rng.randrange(1 if rng.random() < 0.1 else low, capacity + 1) for _ in range(batch)]
        return _case("decode", batch, layers, kv_heads, capacity, " ".join(map(str, lens)), group=group, kind=kind, block=block)
    if op in ("prefill", "mass") and (op == "prefill" or rng.random() < 0.4):
        batch = _log_int(rng, 1, 3)
        n_new = _log_int(rng, 2, min(1024, capacity // 2))
        lens = [rng.randrange(max(n_new, low), capacity + 1) for _ in range(batch)]
        layers = rng.randrange(1, 3)
        if op == "prefill":
            return _case("prefill", batch, layers, min(kv_heads, 8), capacity, " ".join(map(str, lens)), group=group, n_new=n_new, kind=kind,
                         block=block)
        return _case("mass", batch, layers, min(kv_heads, 8), capacity, " ".join(map(str, lens)), group=group, n_new=n_new, dtype="bf16")
    if op == "mass":
        batch, layers = _log_int(rng, 1, 8), rng.randrange(1, 5)
        lens = [rng.randrange(low, capacity + 1) for _ in range(batch)]
        return _case("mass", batch, layers, kv_heads, capacity, " ".join(map(str, lens)), group=group, n_new=1,
                     dtype=rng.choice(["bf16", "bf16", "fp32"]))
    batch, layers = _log_int(rng, 1, 8), rng.randrange(1, 9)
    sink = rng.choice([0, 4, 4, rng.randrange(1, 17)])
    lens = [rng.randrange(low + sink, capacity + 1) for _ in range(batch)]
    kept = [max(1, int(rng.uniform(0.2, 0.9) * (n - sink))) for n in lens]
    recent = rng.randrange(0, min(kept) + 1)
    return _case("evict", batch, layers, min(kv_heads, 8), capacity, " ".join(map(str, lens)), kept=" ".join(map(str, kept)), sink=sink,
                 recent=recent, dtype=rng.choice(["bf16", "bf16", "fp32"]))


def _ints(case, key):
    got = [int(x) for x in case[key].split()]
    return got * case["batch"] if len(got) == 1 else got


def work(case):
    B, L, H, lens = case["batch"], case["layers"], case["kv_heads"], _ints(case, "lens")
    op, G = case["op"], case.get("group", 1)
    if op == "write":
        rows = sum(lens) if case["how"] == "quantize" else B * case["n_new"]
        scales = sum(-(-n // case["block"]) for n in lens) if case["how"] == "quantize" else B * -(-case["n_new"] // case["block"])
        return {"bytes": 2 * L * H * (rows * HEAD * (SRC_BYTES[case["dtype"]] + 1) + 4 * scales), "flops": 2 * L * H * rows * HEAD * 2}
    if op == "evict":
        rows = sum(_ints(case, "kept"))
        return {"bytes": L * H * (rows * HEAD * 4 * SRC_BYTES[case["dtype"]] + 4 * (sum(lens) + 2 * rows)), "flops": L * H * sum(lens)}
    n = case.get("n_new", 1)
    pairs = sum(n * (x - n) + n * (n + 1) // 2 for x in lens) * L * H * G
    rows = sum(lens) * L * H
    if op == "mass":
        e = SRC_BYTES[case["dtype"]]
        io = 8 * rows + B * L * H * G * n * HEAD * e * (2 if n == 1 else 1)
        return {"bytes": rows * HEAD * e * (2 if n == 1 else 1) + io, "flops": (4 if n == 1 else 2) * HEAD * pairs}
    scales = sum(-(-x // case["block"]) for x in lens) * L * H
    return {"bytes": 2 * rows * HEAD + 8 * scales + 2 * B * L * H * G * n * HEAD * 2, "flops": 4 * HEAD * pairs}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _sequences(gen, shape, dtype):
    """Rows [batch, layers, kv_heads, tokens, HEAD]: a moving average along the tokens, per-channel scales, two outlier channels a head."""
    B, L, H, T, D = shape
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for b in range(B):
        x = torch.randn(L, H, T + 7, D, generator=gen, device="cuda")
        y = sum(x[:, :, i:i + T] * (0.436 * 0.9 ** i) for i in range(8))
        scale = torch.rand(L, H, 1, D, generator=gen, device="cuda") * 1.5 + 0.5
        loud = torch.randint(0, D, (L, H, 1, 2), generator=gen, device="cuda")
        out[b] = (y * scale.scatter(3, loud, scale.gather(3, loud) * 8)).to(dtype)
    return out


def _mass_values(gen, shape):
    """Accumulated weights as they come out of attention: heavy-tailed, a few rows far above the others."""
    return (torch.randn(shape, generator=gen, device="cuda") * 1.5 - 3).exp()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    B, L, H, T, lens = case["batch"], case["layers"], case["kv_heads"], case["capacity"], _ints(case, "lens")
    op, G, n = case["op"], case.get("group", 1), case.get("n_new", 1)
    st = dict(case=case, lens=lens, at=torch.tensor(lens, device="cuda"))
    if op == "evict":
        st["k"], st["v"] = (_sequences(gen, (B, L, H, T, HEAD), SRC[case["dtype"]]) for _ in range(2))
        st["mass"] = _mass_values(gen, (B, L, H, T))
        st["mass_out"] = torch.zeros(B, L, H, T, device="cuda")
        st["rows"] = torch.full((B, L, H, T), -1, dtype=torch.int32, device="cuda")
        st["kept"] = _ints(case, "kept")
        st["kept_at"] = torch.tensor(st["kept"], device="cuda")
        return st
    if op == "write":
        blocks = -(-T // case["block"])
        st["codes"] = [torch.zeros(B, L, H, T, HEAD, dtype=torch.int8, device="cuda").view(CODES[case["kind"]]) for _ in range(2)]
        st["scales"] = [torch.zeros(B, L, H, blocks, device="cuda") for _ in range(2)]
        if case["how"] == "quantize":
            st["new"] = [_sequences(gen, (B, L, H, T, HEAD), SRC[case["dtype"]]) for _ in range(2)]
        else:
            old = [_sequences(gen, (B, L, H, T, HEAD), torch.bfloat16) for _ in range(2)]
            for i in range(2):
                _quantize_into(old[i], st["codes"][i], st["scales"][i], st["at"], case["kind"], case["block"])
            st["new"] = [_sequences(gen, (B, L, H, n, HEAD), SRC[case["dtype"]]) for _ in range(2)]
            # the rows of all blocks that the new rows touch, up to the last new one: (sequence, row) and what row of the window it is
            first = [x // case["block"] * case["block"] for x in lens]
            st["window"] = -(-max(x + n - f for x, f in zip(lens, first)) // case["block"])
            pairs = [(b, r) for b in range(B) for r in range(first[b], lens[b] + n)]
            st["touched"] = torch.tensor([(b, r, r - first[b]) for b, r in pairs], device="cuda").T.contiguous()
            st["first"] = torch.tensor(first, device="cuda")
        return st
    if op == "mass":
        st["k"], st["v"] = (_sequences(gen, (B, L, H, T, HEAD), SRC[case["dtype"]]) for _ in range(2))
        st["mass"] = _mass_values(gen, (B, L, H, T)) / T
    else:
        st["codes"], st["scales"] = [], []
        for _ in range(2):
            rows = _sequences(gen, (B, L, H, T, HEAD), torch.bfloat16)
            codes = torch.zeros(B, L, H, T, HEAD, dtype=torch.int8, device="cuda").view(CODES[case["kind"]])
            scales = torch.zeros(B, L, H, -(-T // case["block"]), device="cuda")
            _quantize_into(rows, codes, scales, torch.full_like(st["at"], T), case["kind"], case["block"])
            st["codes"].append(codes)
            st["scales"].append(scales)
    dtype = SRC[case.get("dtype", "bf16")]
    shape = (L, B, H * G, HEAD) if op == "decode" or (op == "mass" and n == 1) else (L, B, H * G, n, HEAD)
    st["q"] = torch.randn(shape, generator=gen, device="cuda").to(dtype)
    st["out"] = torch.empty_like(st["q"])
    return st


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _scale_of(largest, kind):
    """The scale of a block whose largest magnitude is given."""
    if kind == "int8":
        s = (largest.double() / 127).float()
    else:
        m, e = torch.frexp(largest)                      # largest = m 2^e, m in [0.5, 1): 448 = 0.875 * 2^9
        s = torch.ldexp(torch.ones_like(m), e - 9 + (m > 0.875).int())
    return torch.where(largest > 0, s.clamp(min=TINY), torch.zeros_like(s))


def _codes(x, s, kind):
    """Codes of the values x under the scales s: the quotient in 64 bits, rounded once, ties to even."""
    t = x.double() / torch.where(s > 0, s, torch.ones_like(s)).double()
    if kind == "int8":
        return t.round_().clamp_(-127, 127).to(torch.int8)
    return t.clamp_(-448, 448).float().to(torch.float8_e4m3fn)


def _quantize_into(x, codes, scales, lens, kind, block):
    """Rows [0, lens) of x [B, L, H, T, D] as codes and block scales; other rows and scales stay.  T is a multiple of the block."""
    B, L, H, T, D = x.shape
    nb = T // block
    row = torch.arange(T, device=x.device)
    live = row < lens[:, None]                                              # [B, T]
    largest = torch.where(live[:, None, None, :, None], x.float().abs(), 0).view(B, L, H, nb, block * D).amax(4)
    s = _scale_of(largest, kind)
    new = _codes(x.view(B, L, H, nb, block, D), s[..., None, None], kind).view(B, L, H, T, D)
    codes.view(torch.int8).copy_(torch.where(live[:, None, None, :, None], new.view(torch.int8), codes.view(torch.int8)))
    touched = (torch.arange(nb, device=x.device) * block < lens[:, None])[:, None, None]
    scales.copy_(torch.where(touched, s, scales))


def _append_into(x, codes, scales, st):
    """Rows x [B, L, H, n, D] enter behind the first lens rows of every sequence."""
    case, lens, first, W = st["case"], st["at"], st["first"], st["window"]
    B, L, H, n, D = x.shape
    block, kind, T = case["block"], case["kind"], codes.shape[3]
    b, r, w = st["touched"]
    is_new = r >= lens[b]
    # all touched rows of a sequence in a window of whole blocks, [B, W * block, L, H, D]; rows past the last one stay zero
    fresh = torch.zeros(B, W * block, L, H, D, device=x.device)
    fresh[b, w] = torch.where(is_new[:, None, None, None], x.float().permute(0, 3, 1, 2, 4)[b, (r - lens[b]).clamp(min=0)], 0.0)
    largest = fresh.abs().view(B, W, block, L, H, D).amax((2, 5))           # [B, W, L, H]
    blk = first[:, None] // block + torch.arange(W, device=x.device)
    inside = blk * block < T
    had = scales.permute(0, 3, 1, 2)[torch.arange(B, device=x.device)[:, None], blk.clamp(max=scales.shape[3] - 1)]
    had = torch.where((blk * block < lens[:, None])[..., None, None], had, 0.0)
    s = torch.maximum(had, _scale_of(largest, kind))
    old = codes.view(torch.int8).permute(0, 3, 1, 2, 4)[b, r].view(CODES[kind])
    at = w // block
    value = torch.where(is_new[:, None, None, None], fresh[b, w].double(), old.to(torch.float32).double() * had[b, at][..., None].double())
    codes.view(torch.int8).permute(0, 3, 1, 2, 4)[b, r] = _codes(value, s[b, at][..., None], kind).view(torch.int8)
    used = inside & (blk * block < (lens + n)[:, None])
    put = blk.clamp(max=scales.shape[3] - 1)
    keep = torch.zeros(B, scales.shape[3], dtype=torch.int32, device=x.device).scatter_add_(1, put, used.int()) > 0
    full = torch.zeros(B, scales.shape[3], L, H, device=x.device).scatter_add_(1, put[..., None, None].expand(B, W, L, H),
                                                                             torch.where(used[..., None, None], s, 0.0))
    scales.copy_(torch.where(keep[:, None, None], full.permute(0, 2, 3, 1), scales))


def _values(codes, scales, block):
    B, L, H, T, D = codes.shape
    return (codes.to(torch.float32).view(B, L, H, T // block, block, D) * scales[..., None, None]).view(B, L, H, T, D)


def _rotate(x, pos):
    """Channel pairs (c, c + 64) of x [..., HEAD] turned by pos * BASE^(-2c / HEAD); pos broadcasts against x's leading axes."""
    angle = pos.double()[..., None] * BASE ** (-torch.arange(HEAD // 2, device=x.device).double() * 2 / HEAD)
    c, s = angle.cos().float(), angle.sin().float()
    lo, hi = x[..., :HEAD // 2], x[..., HEAD // 2:]
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)


def _weights(q, k, lens, n):
    """Softmax weights [B, L, H, G, n, T] of queries [L, B, heads, n, D] at rows lens - n + i over rows [0, lens - n + i] of k."""
    L, B, heads, _, D = q.shape
    H, T = k.shape[2], k.shape[3]
    pos = lens[:, None] - n + torch.arange(n, device=q.device)              # [B, n]
    q = _rotate(q.float(), pos[:, None]).transpose(0, 1).reshape(B, L, H, heads // H * n, D)
    k = _rotate(k, torch.arange(T, device=q.device))
    s = ((q @ k.transpose(-1, -2)) * D ** -0.5).view(B, L, H, heads // H, n, T)
    hidden = torch.arange(T, device=q.device) > pos[..., None]              # [B, n, T]
    s.masked_fill_(hidden[:, None, None, None], -math.inf)
    s -= s.amax(-1, keepdim=True)
    s.exp_()
    return s.div_(s.sum(-1, keepdim=True))


def _weighted(w, v):
    """Weighted values as queries are laid out: [L, B, heads, n, D]."""
    B, L, H, G, n, T = w.shape
    return (w.view(B, L, H, G * n, T) @ v).view(B, L, H * G, n, -1).transpose(0, 1)


def _evict_plain(st):
    case, mass, lens = st["case"], st["mass"], st["at"][:, None, None, None]
    sink, recent, T = case["sink"], case["recent"], mass.shape[3]
    row = torch.arange(T, device=mass.device).expand(mass.shape)
    open_ = (row >= sink) & (row < lens - recent)
    order = torch.where(open_, mass, -math.inf).sort(dim=3, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(3, order, row)
    heavy = st["kept_at"][:, None, None, None] - recent
    keep = (open_ & (rank < heavy)) | (row < sink) | ((row >= lens - recent) & (row < lens))
    most = sink + max(st["kept"])
    rows = torch.where(keep, row, T).sort(dim=3)[0][..., :most]
    fits = rows < T
    rows = rows.clamp(max=T - 1)
    for x in (st["k"], st["v"]):
        moved = x.gather(3, rows[..., None].expand(*rows.shape, x.shape[4]))
        x[:, :, :, :most] = torch.where(fits[..., None], moved, x[:, :, :, :most])
    st["mass_out"].copy_(torch.where(row < lens, 0.0, st["mass_out"]))
    st["mass_out"][..., :most] = torch.where(fits, mass.gather(3, rows), st["mass_out"][..., :most])
    st["rows"][..., :most] = torch.where(fits, rows.int(), st["rows"][..., :most])
    return st["k"], st["v"], st["mass_out"], st["rows"]


def _run_plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "evict":
        return _evict_plain(st)
    if op == "write":
        for x, codes, scales in zip(st["new"], st["codes"], st["scales"]):
            if case["how"] == "quantize":
                _quantize_into(x, codes, scales, st["at"], case["kind"], case["block"])
            else:
                _append_into(x, codes, scales, st)
        return st["codes"], st["scales"]
    q, n = st["q"], case.get("n_new", 1)
    rows = q if q.dim() == 5 else q.unsqueeze(3)
    if op == "mass":
        w = _weights(rows, st["k"].float(), st["at"], n)
        st["mass"] += w.sum((3, 4))
        if n > 1:
            return st["mass"]
        return _weighted(w, st["v"].float()).view_as(q).to(q.dtype), st["mass"]
    k, v = (_values(c, s, case["block"]) for c, s in zip(st["codes"], st["scales"]))
    return _weighted(_weights(rows, k, st["at"], n), v).view_as(q).to(q.dtype)


# ---- the library's calls ----------------------------------------------------------------------------------------------

_contexts = []


def _context():
    from paper_2505_00570_b200 import binding as fk

    if not _contexts:
        _contexts.append(fk.Context())
    return fk, _contexts[0]


def _run_own(st):
    fk, ctx = _context()
    case, op, lens = st["case"], st["case"]["op"], st["lens"]
    if op == "evict":
        ctx.evict(st["k"], st["v"], st["mass"], lens, st["kept"], case["sink"], case["recent"], mass_out=st["mass_out"], kept_rows=st["rows"])
        return st["k"], st["v"], st["mass_out"], st["rows"]
    if op == "mass":
        if case["n_new"] > 1:
            for layer in range(case["layers"]):
                ctx.attend_mass(st["k"], layer, st["q"][layer], st["mass"], lens, rope_base=BASE)
            return st["mass"]
        for layer in range(case["layers"]):
            ctx.attend_decode_mass(st["k"], st["v"], layer, st["q"][layer], st["mass"], lens, rope_base=BASE, out=st["out"][layer])
        return st["out"], st["mass"]
    cache = fk.Q8Cache(*st["codes"], *st["scales"], case["block"])
    if op == "write":
        if case["how"] == "quantize":
            ctx.quantize(*st["new"], lens, cache)
        else:
            ctx.append_q8(cache, *st["new"], lens)
        return st["codes"], st["scales"]
    attend = ctx.attend_decode_q8 if op == "decode" else ctx.attend_prefill_q8
    for layer in range(case["layers"]):
        attend(cache, layer, st["q"][layer], lens, rope_base=BASE, out=st["out"][layer])
    return st["out"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- 64 bits ------------------------------------------------------------------------------------------------------------

def _exact_block(rows, first, old, s_old, kind):
    """One block's codes (as numbers) and scale: old codes rows [0, first), then the values rows; all layers and heads at once."""
    big = rows.double().abs().amax((2, 3)) if rows.shape[2] else torch.zeros(rows.shape[:2], dtype=torch.float64, device=rows.device)
    if kind == "int8":
        s = (big / 127).float().double()
    else:
        s = torch.exp2(torch.ceil(torch.log2(big.clamp(min=1e-300) / 448)))
        s = torch.where(big <= 224 * s, s / 2, s)        # a logarithm that came out a hair too high
        s = torch.where(big > 448 * s, s * 2, s)
    s = torch.where(big > 0, s.clamp(min=TINY), 0.0)
    if first:
        s = torch.maximum(s, s_old.double())
        rows = torch.cat((old.double() * s_old.double()[..., None, None], rows.double()), 2)
    t = rows.double() / torch.where(s > 0, s, 1.0)[..., None, None]
    if kind == "int8":
        return torch.round(t), s
    # steps of a binary floating format of 4 significant bits whose smallest normal number is 2^-6
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(t / step) * step, s


def _exact_write(case, st):
    block, n = case["block"], case["n_new"]
    codes = [c.to(torch.float32).double() for c in st["codes"]]
    scales = [s.double() for s in st["scales"]]
    for i in range(2):
        for b, had in enumerate(st["lens"]):
            start, end = (0, had) if case["how"] == "quantize" else (had, had + n)
            at = start // block * block
            while at < end:
                lo, hi = max(start, at), min(end, at + block)
                src = st["new"][i][b, :, :, lo - (0 if case["how"] == "quantize" else had):][:, :, :hi - lo]
                c, s = _exact_block(src, lo - at, codes[i][b, :, :, at:lo], scales[i][b, :, :, at // block], case["kind"])
                codes[i][b, :, :, at:hi], scales[i][b, :, :, at // block] = c, s
                at += block
    return [None, None] if case["kind"] == "int8" else codes, scales


def _exact_attention(q, k, v, length, n):
    """One sequence and layer, q [heads, n, D], k, v [H, length, D]: weighted values [heads, n, D], weights summed a KV head [H, length]."""
    H, T, D = k.shape
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=q.device), torch.arange(T, device=q.device).double()[:, None] *
                       torch.exp(-math.log(BASE) * torch.arange(D // 2, device=q.device).double() / (D // 2)))
    zk = torch.complex(k[..., :D // 2].double(), k[..., D // 2:].double()) * turn
    zq = torch.complex(q[..., :D // 2].double(), q[..., D // 2:].double()) * turn[T - n:]
    out, total = [], []
    for h in range(H):
        mine = slice(h * (q.shape[0] // H), (h + 1) * (q.shape[0] // H))
        s = (zq[mine] @ zk[h].conj().T).real / math.sqrt(D)
        s = s + torch.full((n, T), -math.inf, dtype=torch.float64, device=q.device).triu(T - n + 1)
        p = torch.softmax(s, -1)
        out.append(p @ v[h].double())
        total.append(p.sum((0, 1)))
    return torch.cat(out), torch.stack(total)


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "write":
        return _exact_write(case, st)
    if op == "evict":
        return _exact_evict(case, st)
    n, q = case.get("n_new", 1), st["q"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    mass = st["mass"].double() if op == "mass" else None
    for layer in range(case["layers"]):
        for b, length in enumerate(st["lens"]):
            if op == "mass":
                k, v = st["k"][b, layer, :, :length], st["v"][b, layer, :, :length]
            else:
                k, v = (c[b, layer, :, :length].to(torch.float32).double() *
                        s[b, layer].double().repeat_interleave(case["block"], 1)[:, :length, None] for c, s in zip(st["codes"], st["scales"]))
            o, w = _exact_attention(q[layer, b].reshape(q.shape[2], n, HEAD), k, v, length, n)
            out[layer, b] = o.view_as(out[layer, b])
            if op == "mass":
                mass[b, layer, :, :length] += w
    if op == "mass":
        return mass if n > 1 else (out, mass)
    return out


def _exact_evict(case, st):
    sink, recent = case["sink"], case["recent"]
    k, v, mass = st["k"].clone(), st["v"].clone(), st["mass_out"].double()
    for b, (length, kept) in enumerate(zip(st["lens"], st["kept"])):
        m = st["mass"][b, :, :, sink:length - recent].double()
        top = torch.sort(torch.argsort(-m, dim=-1, stable=True)[..., :kept - recent], dim=-1)[0] + sink
        ends = [torch.arange(x, y, device="cuda").expand(*m.shape[:2], y - x) for x, y in ((0, sink), (length - recent, length))]
        rows = torch.cat((ends[0], top, ends[1]), -1)
        for x, y in ((k, st["k"]), (v, st["v"])):
            x[b, :, :, :sink + kept] = torch.take_along_dim(y[b], rows[..., None], 2)
        mass[b, :, :, :length] = 0
        mass[b, :, :, :sink + kept] = torch.take_along_dim(st["mass"][b], rows, 2).double()
    return k, v, mass, None
