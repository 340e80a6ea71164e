"""Operator cases: a key/value cache held in 4 bits, and the attention over it.

An attention context model decodes a latent grid in the same wavefront order as
the convolutional one: after each step the new latents' keys and values join a
cache, and the next step's queries attend to everything decoded before.  The
cache is what such a decoder reads most, so it is held in 4 bits.  Operators:

  write   wf.Cache.write: keys and values are quantised as they enter the
          cache's pages.  A pass writes and reads the same tokens back, as an
          encoder does to see exactly the values its decoder will
  read    wf.Cache.read: cached tokens as the values they stand for
  attend  wf.Cache.attend: softmax(scale q k^T) v over the cached tokens of
          each sequence; shared heads (q_heads a multiple of heads), one
          prefix length for each query row, an optional mask

Format: a block of 32 consecutive channels of one token's head holds 4-bit
values {0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign, times a power of two of its
own.  The power is the smallest 2^e, -125 <= e <= 125, with 6 * 2^e >= the
block's largest magnitude; values are rounded to the nearest, a tie to the even
code.  A block that holds a value that is not finite reads back as NaN.

Sizes: latent grids of inputs.WORKLOADS (256, 1536, 8160 and 32400 latents; 192
and 320 channels as heads of 64) and generic serving shapes.
"""
import math
import random

import torch

own = False

BLOCK = 32
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
#: attended (row, key, channel) triples and cached values of the largest case
MOST_PAIRS, MOST_VALUES = 32 * 1024 * 16384 * 128, 64 * 8192 * 8 * 128


def _case(name, op, B, n, heads, dim, dtype, len, q_heads=0, ragged=False, causal=False, mask=False, fused=False,
          page=64):
    return {"name": name, "op": op, "B": B, "n": n, "heads": heads, "dim": dim, "dtype": dtype, "len": len,
            "q_heads": q_heads or heads, "ragged": ragged, "causal": causal, "mask": mask, "fused": fused,
            "page": page}


def listed():
    return [
        # a decoder's step for one sequence: one token joins a cache of 1001
        _case("write_token", "write", 1, 1, 8, 128, "bf16", 1001),
        # a batch of images, up to 45 latents each in a wavefront step, 320 channels
        _case("write_step_ragged_fp32", "write", 8, 45, 5, 64, "fp32", 8160, ragged=True),
        # two prompts, keys and values taken as views of the fused projection's output
        _case("write_prompt_fused", "write", 2, 8191, 8, 128, "bf16", 8191, fused=True),
        # the cache of a 256x256 image, 192 channels
        _case("read_16x16_fp32", "read", 1, 256, 3, 64, "fp32", 256),
        # four 4K images' latents, read back whole
        _case("read_4k_b4", "read", 4, 32400, 5, 64, "bf16", 32400),
        # one token of one short sequence: the call's latency
        _case("token_short", "attend", 1, 1, 8, 128, "bf16", 1001, q_heads=32),
        # one token of one long sequence: the long axis is all there is to share out
        _case("token_long", "attend", 1, 1, 8, 128, "bf16", 131072, q_heads=32),
        # one token each of 64 sequences of unequal length
        _case("token_batch_ragged", "attend", 64, 1, 8, 128, "bf16", 8192, q_heads=32, ragged=True),
        # a wavefront step near the end of a 4K grid, 320 channels, fp32, no shared heads
        _case("step_4k_fp32", "attend", 1, 45, 5, 64, "fp32", 32300),
        # a step that sees part of the grid: a mask that leaves some rows nothing, odd sizes
        _case("step_masked", "attend", 2, 34, 2, 96, "bf16", 8101, q_heads=6, mask=True),
        # wide heads, all queries on one key head, fp32
        _case("rows_dim256_fp32", "attend", 4, 7, 1, 256, "fp32", 20011, q_heads=8, causal=True, page=32),
        # a chunk of a long prompt, each row seeing those before it
        _case("chunk_causal", "attend", 1, 1024, 8, 128, "bf16", 16384, q_heads=32, causal=True, fused=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["write", "read", "attend", "attend", "attend", "attend"])
    heads, dim = rng.choice([1, 2, 3, 5, 8]), rng.choice([40, 64, 64, 96, 128, 128, 128, 256])
    B = _log_int(rng, 1, 64)
    room = MOST_VALUES // (B * heads * dim)
    c = {"op": op, "B": B, "heads": heads, "dim": dim, "dtype": rng.choice(["bf16", "bf16", "fp32"]),
         "page": rng.choice([32, 64, 64, 128]), "ragged": rng.random() < 0.4, "fused": rng.random() < 0.3,
         "q_heads": heads, "causal": False, "mask": False}
    if op != "attend":
        c["n"] = _log_int(rng, 1, min(32400, max(1, room // 8)))
        c["len"] = c["n"] + rng.randint(0, 300)
        return c
    c["q_heads"] = heads * rng.choice([1, 1, 2, 4, 7, 8])
    c["len"] = _log_int(rng, 40, min(131072, max(40, room)))
    c["n"] = 1 if rng.random() < 0.5 else _log_int(rng, 2, 1024)
    c["n"] = max(1, min(c["n"], c["len"], MOST_PAIRS // (B * c["q_heads"] * c["len"] * dim)))
    c["causal"] = rng.random() < 0.5
    c["mask"] = c["n"] * B * c["len"] <= 1 << 26 and rng.random() < 0.3
    return c


# ---- sizes that follow from a case alone ---------------------------------------


def _lengths(c):
    """Tokens of each sequence: the first has the case's, and where lengths are
    unequal the others a part of it, one in seven none (a slot that waits)."""
    if not c["ragged"]:
        return [c["len"]] * c["B"]
    r = random.Random("%d of %d" % (c["B"], c["len"]))
    return [c["len"]] + [0 if b % 7 == 3 else r.randint(c["len"] // 4, c["len"]) for b in range(1, c["B"])]


def _counts(c):
    """Tokens that each sequence writes or reads."""
    return [min(c["n"], n) for n in _lengths(c)]


def _visible(c):
    """Tokens that each query row sees, [B][n]."""
    return [[max(0, n - (c["n"] - 1 - i if c["causal"] else 0)) for i in range(c["n"])] for n in _lengths(c)]


def work(case):
    c = case
    item = 4 if c["dtype"] == "fp32" else 2
    held = c["dim"] / 2 + -(-c["dim"] // BLOCK)     # bytes of one token's key (or value) of one head
    if c["op"] != "attend":
        tokens = sum(_counts(c)) * c["heads"] * 2
        passes = 2 if c["op"] == "write" else 1
        return {"bytes": tokens * passes * (held + c["dim"] * item), "flops": 4.0 * tokens * passes * c["dim"]}
    seen = _visible(c)
    kept = 0.4 if c["mask"] else 1.0                # half of each row, one row in five empty
    pairs = sum(map(sum, seen)) * kept
    return {"bytes": sum(map(max, seen)) * c["heads"] * 2 * held + 2.0 * c["B"] * c["n"] * c["q_heads"] * c["dim"] * item
            + (c["B"] * c["n"] * c["len"] if c["mask"] else 0),
            "flops": 4.0 * pairs * c["q_heads"] * c["dim"]}


# ---- inputs -----------------------------------------------------------------------


def _inputs(c, seed):
    """What a pass is given, as tensors on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = DTYPES[c["dtype"]]
    B, H, D, L = c["B"], c["heads"], c["dim"], c["len"]
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    # some channels of keys are several times larger than the rest, and keys have an offset
    spread = torch.exp(0.5 * normal(H, D))
    offset = 0.5 * normal(H, D)
    attend = c["op"] == "attend"
    T = L if attend else c["n"]
    Hq = c["q_heads"] if attend else 0
    q = 2.0 * normal(B, c["n"], Hq, D) if attend else None
    if c["fused"] and not attend:
        both = torch.empty((B, T, 2 * H, D), device="cuda", dtype=dtype)
        k, v = both[:, :, :H], both[:, :, H:]
        k.copy_(normal(B, T, H, D) * spread + offset)
        v.copy_(normal(B, T, H, D))
    else:
        k, v = (normal(B, T, H, D) * spread + offset).to(dtype), normal(B, T, H, D).to(dtype)
    if attend:
        q = (q / spread.repeat_interleave(Hq // H, 0)).to(dtype)
        if c["fused"]:
            wide = torch.empty((B, c["n"], Hq + 2 * H, D), device="cuda", dtype=dtype)
            wide[:, :, :Hq] = q
            q = wide[:, :, :Hq]
    per = -(-L // c["page"])
    table = torch.randperm(B * per, generator=g, device="cuda").to(torch.int32).reshape(B, per)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lengths = _lengths(c)
    counts = lengths if attend else _counts(c)
    # a cache is filled from its start; tokens that are written or read are its last
    first = [0] * B if attend else [n - m for n, m in zip(lengths, counts)]
    d = {"q": q, "k": k, "v": v, "table": table, "first": ints(first), "counts": ints(counts), "mask": None}
    if attend:
        d["visible"] = ints(_visible(c))
        if c["mask"]:
            d["mask"] = torch.rand((B, c["n"], L), generator=g, device="cuda") < 0.5
            d["mask"][:, 4::5] = False
    return d


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    s["cache"] = _cache(c["heads"], c["dim"], s["table"].numel(), c["page"])
    if c["op"] != "write":      # a program that reads or attends has filled the cache before
        s["cache"].write(s.pop("k"), s.pop("v"), s["table"], s["first"], counts=s["counts"])
    return s


def run(state):
    s, c = state, state["case"]
    if c["op"] == "attend":
        return s["cache"].attend(s["q"], s["table"], s["visible"], mask=s["mask"], max_visible=c["len"])
    if c["op"] == "write":
        s["cache"].write(s["k"], s["v"], s["table"], s["first"], counts=s["counts"])
    return s["cache"].read(s["table"], s["first"], c["n"], counts=s["counts"], dtype=DTYPES[c["dtype"]])


def _cache(heads, dim, pages, page):
    if own:
        from paper_2607_19082_amd import wf
        return wf.Cache(heads, dim, pages, page=page)
    return Plain(heads, dim, pages, page)


# ---- the plain form ------------------------------------------------------------------


def _power(e):
    """2^e in 32 bits, from its exponent bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


class Plain:
    """The cache and its operators in elementary torch operations, in 32 bits."""

    def __init__(self, heads, dim, pages, page):
        self.heads, self.dim, self.page = heads, dim, page
        self.blocks = -(-dim // BLOCK)
        slots = pages * page + 1        # the last takes tokens that are not to be written
        self.codes = torch.zeros((2, slots, heads, self.blocks * BLOCK // 2), dtype=torch.uint8, device="cuda")
        self.powers = torch.zeros((2, slots, heads, self.blocks), dtype=torch.uint8, device="cuda")

    def _slots(self, table, first, n, counts):
        i = torch.arange(n, device="cuda")
        at = first[:, None] + i
        slot = table.gather(1, (at // self.page).clamp(max=table.shape[1] - 1).long()) * self.page + at % self.page
        inside = i < counts[:, None]
        return torch.where(inside, slot, self.codes.shape[1] - 1).long(), inside

    def write(self, k, v, table, first, counts):
        slot, _ = self._slots(table, first, k.shape[1], counts)
        x = torch.stack([k, v]).float()
        x = torch.nn.functional.pad(x, (0, self.blocks * BLOCK - self.dim)).unflatten(-1, (self.blocks, BLOCK))
        top = x.abs().amax(-1)
        f, e = torch.frexp(top)         # top = f 2^e with 1/2 <= f < 1, and 6 = 3/4 2^3
        e = torch.where(f <= 0.75, e - 3, e - 2).clamp(-125, 125)
        e = torch.where(top == 0, -125, e)
        y = x * _power(-e)[..., None]
        a = y.abs()
        code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte()
                + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5.0).byte())
        code = (code + 8 * (y < 0).byte()).flatten(-2)
        self.codes[:, slot] = code[..., 0::2] + 16 * code[..., 1::2]
        self.powers[:, slot] = torch.where(torch.isfinite(top), e + 127, 255).byte()

    def _values(self, slot):
        """Keys and values of the slots, [2][..., heads][dim] in 32 bits."""
        packed, power = self.codes[:, slot], self.powers[:, slot].int()
        code = torch.stack([packed & 15, packed >> 4], -1).flatten(-2)
        m = (code & 7).float()
        x = torch.where(m < 4, 0.5 * m, torch.where(m < 6, m - 2.0, 2.0 * m - 8.0))
        x = torch.where(code >= 8, -x, x).unflatten(-1, (self.blocks, BLOCK))
        scale = torch.where(power == 255, math.nan, _power(power - 127))
        return (x * scale[..., None]).flatten(-2)[..., :self.dim]

    def read(self, table, first, n, counts, dtype):
        slot, inside = self._slots(table, first, n, counts)
        x = torch.where(inside[..., None, None], self._values(slot), 0.0).to(dtype)
        return x[0], x[1]

    def attend(self, q, table, visible, mask, max_visible):
        B, n, Hq, D = q.shape
        H = self.heads
        slot, _ = self._slots(table, torch.zeros_like(visible[:, 0]), max_visible, visible.amax(1))
        k, v = self._values(slot).transpose(2, 3)                             # [B][H][L][D]
        rows = q.float().unflatten(2, (H, Hq // H)).permute(0, 2, 1, 3, 4).flatten(2, 3)
        s = torch.matmul(rows, k.transpose(2, 3).contiguous()) * (D ** -0.5)  # [B][H][n G][L]
        see = torch.arange(max_visible, device="cuda") < visible[..., None]
        if mask is not None:
            see = see & mask
        see = see.repeat_interleave(Hq // H, 1)[:, None]
        s = torch.where(see, s, -math.inf)
        p = torch.where(see, torch.exp(s - s.amax(-1, keepdim=True)), 0.0)
        total = p.sum(-1, keepdim=True)
        v = torch.where(see.any(2)[..., None], v, 0.0)
        o = torch.matmul(p / torch.where(total == 0, 1.0, total), v)
        return o.unflatten(2, (n, Hq // H)).permute(0, 2, 1, 3, 4).flatten(2, 3).to(q.dtype)


# ---- the definition in 64 bits -----------------------------------------------------------


def _rounded(x):
    """The values that the cache holds for x [..., D], from the definition, in 64 bits."""
    D = x.shape[-1]
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for d in range(0, D, BLOCK):
        b = x[..., d:d + BLOCK].double()
        top = b.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 6.0))
        # the logarithm's own rounding: step to the smallest power that holds the block
        two = lambda n: ((n.long() + 1023) << 52).view(torch.float64)  # noqa: E731
        e = torch.where(torch.isfinite(e), e, 0.0)
        e = torch.where(6.0 * two(e) < top, e + 1, e)
        e = torch.where(6.0 * two(e - 1) >= top, e - 1, e).clamp(-125, 125)
        power = two(e)
        y = (b / power).abs()
        step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
        y = (torch.round(y / step) * step).clamp(max=6.0) * torch.sign(b) * power
        out[..., d:d + BLOCK] = torch.where(torch.isfinite(top), y, math.nan)
    return out


def exact(case, seed):
    c = case
    d = _inputs(c, seed)
    if c["op"] != "attend":
        inside = (torch.arange(c["n"], device="cuda") < d["counts"][:, None])[..., None, None]
        return tuple(torch.where(inside, _rounded(d[x]), 0.0) for x in ("k", "v"))
    B, n, Hq, D = d["q"].shape
    out = torch.zeros((B, n, Hq, D), dtype=torch.float64, device="cuda")
    seen, G = _visible(c), Hq // c["heads"]
    for b in range(B):
        L = max(seen[b])
        if not L:
            continue
        see = torch.arange(L, device="cuda") < d["visible"][b][:, None]
        if c["mask"]:
            see &= d["mask"][b, :, :L]
        for h in range(c["heads"]):
            k, v = _rounded(d["k"][b, :L, h]), _rounded(d["v"][b, :L, h])
            for g in range(h * G, h * G + G):
                s = torch.mm(d["q"][b, :, g].double(), k.t().contiguous()) / math.sqrt(D)
                s.masked_fill_(~see, -math.inf)
                w = torch.softmax(s, -1)
                w.masked_fill_(~see, 0.0)
                out[b, :, g] = torch.mm(w, v)
    return out
