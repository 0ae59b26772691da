"""Decoding in 4 bits, as measurable cases.

Four operators, reached through the package's entry points:

  proj    ld_gemm_w4: the projection of a few rows by weights in 4 bits, with
          the pre-norm of its rows, the residual or the feed-forward activation
  store   ld_kv4_store of the key/value columns of new rows, and ld_kv4_load
          of the rows around them: the values the cache then stands for
  attn    ld_attn_decode_kv4: queries of 1 to 8 new rows per sequence over a
          4-bit key/value cache; with "sums", each position's attention weight
          is added to its running sum
  evict   ld_kv4_evict: of each head the positions with the largest sums and
          the last ones go into a smaller cache, and ld_kv4_load of it

A 4-bit float (e2m1) is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; with a
power of two 2^e (e >= -100, held as the byte e + 127) for 32 neighbours, the
smallest with max|x| <= 6 2^e.  A 4-bit integer (weights only) is a sign and
0 .. 7, with a bfloat16 scale for a group of 32, 64 or 128 neighbours,
max|w| / 7 rounded to nearest.  Codes are rounded to nearest, ties to even.

Weights [N, K]: [ceil(N / 8)][ceil(K / 256)][64 lanes][4 dwords]; lane 16 g + 8 h + r,
dword s holds row 8 t + r at k = 256 c + 128 h + 32 s + 8 g + e, e < 8: e2m1 in
nibble e; integers with e < 4 as bits 8 e .. 8 e + 2 and the sign in 8 e + 7, the
others (i = e - 4) as bits 8 i + 4 .. 8 i + 6 and the sign in (8 i + 11) mod 32.
Scales [ceil(N / 8)][ceil(K / 256)][2 (h)][8 (r)][128 / group].

Cache of one (sequence, key/value head), S8 being the positions rounded up to 8:
keys [S8][dh / 2] bytes, dimension 2 i in the low nibble of byte i; then values
[S8 / 8][16 (n)][dh / 32 (j)][8 (position)] bytes, dimension 32 j + n low, 32 j + 16 + n
high.  Scales [n_seq][kv_heads][2][S8][dh / 32] bytes.

Ragged cases give each sequence its own position, and leave every fifth out.
"""
import math

import torch

own = False

DEV = "cuda:0"
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MIN_EXP = -100
EPS = 1e-5


# ------------------------------------------------------------------- cases

def _proj(name, fmt, group, m, n, k, act="none", norm=False, resid=False):
    return dict(name=name, kind="proj", fmt=fmt, group=group, m=m, n=n, k=k, act=act, norm=norm, resid=resid)


def _cache(name, kind, n_seq, heads, kv_heads, dh, s_max, pos, n_new, ragged=0, alibi=False, sums=False):
    return dict(name=name, kind=kind, n_seq=n_seq, heads=heads, kv_heads=kv_heads, dh=dh, s_max=s_max, pos=pos,
                n_new=n_new, ragged=ragged, alibi=alibi, sums=sums)


def _evict(name, n_seq, kv_heads, dh, length, keep, recent, ragged=0):
    return dict(name=name, kind="evict", n_seq=n_seq, kv_heads=kv_heads, dh=dh, length=length, keep=keep,
                recent=recent, ragged=ragged)


def listed():
    return [
        # the query/key/value projection of one token of the 125M shape, with
        # its norm: a launch, and little more
        _proj("qkv_125m_b1", "int4", 32, 1, 2304, 768, norm=True),
        # gate, up and SwiGLU of a token of each of 8 sequences of the 1B shape
        _proj("gate_up_1b_b8", "e2m1", 32, 8, 5504, 2048, act="swiglu", norm=True),
        # the down projection of one token of the 7B shape, with its residual
        _proj("down_7b_b1", "int4", 128, 1, 4096, 11008, resid=True),
        # gate, up and SwiGLU of the 7B shape in the verify step of 8 sequences after a draft of five
        _proj("gate_up_7b_verify", "int4", 64, 48, 11008, 4096, act="swiglu"),
        # a decoding step's token for 32 sequences of the 1B shape, each at its own position
        _cache("append_1b_b32", "store", 32, 16, 16, 128, 2056, 2047, 1, ragged=90),
        # prompts of odd length, four query heads to a key/value head
        _cache("prompt_gqa_b3", "store", 3, 32, 8, 128, 1504, 0, 1501),
        # a token over a short cache, the smallest attention
        _cache("attn_125m_b1", "attn", 1, 12, 12, 64, 1024, 199, 1),
        # the verify step after a draft of five, ALiBi, with the positions' weights for a later eviction
        _cache("verify_1b_b8", "attn", 8, 16, 16, 128, 1536, 1500, 6, alibi=True, sums=True),
        # two long contexts, four query heads to a key/value head: little to
        # spread over the chip but the cache's length
        _cache("attn_gqa_long", "attn", 2, 32, 8, 128, 131072, 131071, 1),
        # a serving batch of the 7B shape, lengths from none to 8192
        _cache("attn_7b_b16", "attn", 16, 32, 32, 128, 8192, 8191, 1, ragged=8191),
        # caches of the 1B shape at its training length, cut to a quarter
        _evict("evict_1b_b8", 8, 16, 128, 2048, 512, 64),
        # a long context, few heads
        _evict("evict_gqa_long", 1, 8, 128, 131072, 16384, 1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same kinds and ranges."""
    kind = rng.choice(["proj", "proj", "store", "prompt", "attn", "attn", "evict"])
    if kind == "proj":
        fmt = rng.choice(["e2m1", "int4"])
        group = 32 if fmt == "e2m1" else rng.choice([32, 64, 128])
        m, k, act = _log_int(rng, 1, 64), 8 * _log_int(rng, 8, 2048), rng.choice(["none", "none", "swiglu", "relu2"])
        n = _log_int(rng, 64, 32768)
        while n * k * m > 2 * 11008 * 4096 * 48 // (2 if act == "swiglu" else 1) or n * k > 11008 * 8192:
            n //= 2
        n = -(-n // 8) * 8 if act == "swiglu" else n
        c = _proj("", fmt, group, m, n, k, act, norm=m <= 16 and k <= 8192 and rng.random() < 0.5,
                  resid=act == "none" and rng.random() < 0.5)
        del c["name"]
        return c
    dh = rng.choice([64, 128, 128])
    kv_heads = rng.choice([4, 8, 12, 16, 20, 32])
    n_seq = _log_int(rng, 1, 32)
    if kind == "evict":
        length = _log_int(rng, 200, 100000)
        while n_seq > 1 and n_seq * length * kv_heads * dh > 131072 * 8 * 128:
            n_seq //= 2
        while length * kv_heads * dh > 131072 * 8 * 128:
            length //= 2
        keep = max(17, int(length * rng.uniform(0.05, 0.6)))
        c = _evict("", n_seq, kv_heads, dh, length, keep, rng.choice([0, 1, keep // 8, keep // 2]),
                   rng.choice([0, 0, length]))
        del c["name"]
        return c
    group = rng.choice([1, 1, 1, 2, 4, 8])
    if kind == "prompt":
        n_new, pos, ragged = _log_int(rng, 20, 4000), rng.choice([0, 0, _log_int(rng, 1, 500)]), 0
        most = 8 * 2048 * 16 * 128
    elif kind == "store":
        n_new, pos = rng.randint(1, 8), _log_int(rng, 1, 8000)
        ragged, most = rng.choice([0, min(pos, 100)]), None
    else:
        n_new, pos = rng.choice([1, 1, rng.randint(2, 8)]), _log_int(rng, 30, 100000)
        ragged, most = rng.choice([0, 0, pos]), None
    rows = n_new if most else pos + n_new
    most = most or 2 * 131072 * 8 * 128 // max(1, n_new * group // 16)
    while n_seq > 1 and n_seq * rows * kv_heads * dh > most:
        n_seq //= 2
    while rows * kv_heads * dh > most and kv_heads > 4:
        kv_heads //= 2
    c = _cache("", "store" if kind == "prompt" else kind, n_seq, group * kv_heads, kv_heads, dh,
               pos + n_new + rng.randint(0, 200), pos, n_new, ragged, kind == "attn" and rng.random() < 0.3,
               kind == "attn" and rng.random() < 0.4)
    del c["name"]
    return c


# ------------------------------------------------------------ shared sizes

def _positions(c):
    """Each sequence's first new position: pos, or for ragged cases spread
    over the `ragged` positions before it, with every fifth sequence left out."""
    if not c["ragged"]:
        return [c["pos"]] * c["n_seq"]
    return [-1 if b % 5 == 4 else c["pos"] - (b * 7919) % (c["ragged"] + 1) for b in range(c["n_seq"])]


def _lengths(c):
    """Positions that each sequence of an evict case holds."""
    if not c["ragged"]:
        return [c["length"]] * c["n_seq"]
    return [c["length"] - (b * 7919) % (c["ragged"] + 1) for b in range(c["n_seq"])]


def _window(c):
    """First and last + 1 position that a store case reads back."""
    return min(p for p in _positions(c) if p >= 0), c["pos"] + c["n_new"]


def work(case):
    c = case
    if c["kind"] == "proj":
        rows = c["n"] * (2 if c["act"] == "swiglu" else 1)
        scales = rows * c["k"] / c["group"] * (1 if c["fmt"] == "e2m1" else 2)
        io = c["m"] * (c["k"] + c["n"] * (2 if c["resid"] else 1)) + (c["k"] if c["norm"] else 0)
        return dict(bytes=rows * c["k"] / 2 + scales + 2 * io, flops=2 * c["m"] * rows * c["k"])
    row = c["kv_heads"] * 2 * (c["dh"] / 2 + c["dh"] / 32)   # a position's codes and scales
    wide = c["kv_heads"] * c["dh"] * 4                       # in bfloat16
    if c["kind"] == "evict":
        held = sum(_lengths(c))
        kept = sum(min(n, c["keep"]) for n in _lengths(c))
        # sums in; kept rows, their sums and places; kept rows again, and out in bfloat16
        return dict(bytes=4 * c["kv_heads"] * held + kept * (3 * row + wide + 12 * c["kv_heads"]), flops=0)
    at = [p for p in _positions(c) if p >= 0]
    if c["kind"] == "store":
        lo = _window(c)[0]
        back = sum(p + c["n_new"] - lo for p in at)
        return dict(bytes=len(at) * c["n_new"] * (wide + row) + back * (row + wide), flops=0)
    keys = sum(p + c["n_new"] for p in at)
    pairs = sum(c["n_new"] * (p + (c["n_new"] + 1) / 2) for p in at)
    rows = c["n_seq"] * c["n_new"] * c["heads"] * c["dh"]
    return dict(bytes=keys * row + 2 * rows * 2 + (8 * c["kv_heads"] * keys if c["sums"] else 0),
                flops=4 * c["heads"] * c["dh"] * pairs)


# ------------------------------------------------------------------ inputs

def _need(amax):
    """Exponent e of the smallest 2^e, e >= MIN_EXP, with amax <= 6 2^e."""
    m, e = torch.frexp(amax)                      # amax = m 2^e, m in [1/2, 1); 6 = 0.75 2^3
    e = torch.where(m > 0.75, e + 1, e) - 3
    return torch.where(amax > 0, e, torch.full_like(e, MIN_EXP)).clamp(min=MIN_EXP)


def _to_e2m1(y):
    """Codes of values already divided by their scale: nearest, ties to even."""
    a = y.abs()
    # halfway points between neighbours; an odd code's upper one goes up, an even one's does not
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    return code + 8 * (y < 0).int()


def _from_e2m1(code, dtype=torch.float32):
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=dtype, device=DEV)
    return table[code.long()]


def _quantise(x):
    """e2m1 codes (int32) and scale bytes of the last dimension's groups of 32."""
    x = x.view(*x.shape[:-1], -1, 32)
    e = _need(x.abs().amax(-1))
    code = _to_e2m1(torch.ldexp(x, -e[..., None]))
    return code.flatten(-2), (e + 127).to(torch.uint8)


def _s8(n):
    return (n + 7) // 8 * 8


def _keys(c, codes):
    """Keys' bytes of all positions, [n_seq, kv_heads, S8, dh / 2], as a view of the codes."""
    return codes.view(c["n_seq"], c["kv_heads"], 2, -1, c["dh"] // 2)[:, :, 0]


def _values(c, codes):
    """Values' bytes, [n_seq, kv_heads, S8 / 8, 16, dh / 32, 8], as a view."""
    return codes.view(c["n_seq"], c["kv_heads"], 2, -1, 16, c["dh"] // 32, 8)[:, :, 1]


def _put_keys(code):
    """Bytes of key codes [..., dh]."""
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)


def _put_values(code):
    """Bytes of value codes [..., positions (a multiple of 8), dh]."""
    dh = code.shape[-1]
    x = code.view(*code.shape[:-2], -1, 8, dh // 32, 2, 16)       # tile, position, j, half, n
    b = x[..., 0, :] | (x[..., 1, :] << 4)
    return b.transpose(-1, -3).to(torch.uint8)                    # tile, n, j, position


def _new_cache(c, held, g):
    """A cache whose first held[b] positions are filled."""
    B, KV, dh, s8 = c["n_seq"], c["kv_heads"], c["dh"], _s8(c["s_max"])
    codes = torch.zeros(B * KV * s8 * dh, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(B, KV, 2, s8, dh // 32, dtype=torch.uint8, device=DEV)
    step = max(8, (1 << 24) // (KV * dh) // 8 * 8)
    for b in range(B):
        for p0 in range(0, held[b], step):
            n = min(step, s8 - p0)
            x = (torch.randn(KV, 2, n, dh, device=DEV, generator=g) * 0.9).to(torch.bfloat16).float()
            x[:, :, max(held[b] - p0, 0):] = 0
            code, sc = _quantise(x)
            scales[b, :, :, p0:p0 + n] = sc
            _keys(c, codes)[b, :, p0:p0 + n] = _put_keys(code[:, 0])
            _values(c, codes)[b, :, p0 // 8:(p0 + n) // 8] = _put_values(code[:, 1])
    return codes, scales


def _pack_weights(c, w):
    """Codes (int32 dwords) and scales of w [rows, K] float32."""
    rows, K = w.shape
    T, C = -(-rows // 8), -(-K // 256)
    w = torch.nn.functional.pad(w, (0, 256 * C - K, 0, 8 * T - rows))
    if c["fmt"] == "e2m1":
        code, sc = _quantise(w)
        sc = sc.view(T, 8, C, 2, 4)
        shift = torch.arange(0, 32, 4, device=DEV)
        lay = lambda v: (v << shift).sum(-1)  # noqa: E731
    else:
        x = w.view(8 * T, -1, c["group"])
        s = (x.abs().amax(-1) / 7).clamp(min=2.0 ** MIN_EXP).to(torch.bfloat16)
        q = torch.round(x / s.float()[..., None]).clamp(-7, 7).view(8 * T, -1)
        code = (q.abs().int() | (q < 0).int() << 3)
        sc = s.view(T, 8, C, 2, 128 // c["group"])
        i = torch.arange(4, device=DEV)
        at = torch.cat((8 * i, 8 * i + 4))
        sign = torch.cat((8 * i + 7, (8 * i + 11) % 32))
        lay = lambda v: (((v & 7) << at) | ((v >> 3) << sign)).sum(-1)  # noqa: E731
    # t, r, c, h, s, g, e -> t, c, g, h, r, s, e
    code = code.view(T, 8, C, 2, 4, 4, 8).permute(0, 2, 5, 3, 1, 4, 6).to(torch.int64)
    dwords = lay(code)
    dwords = torch.where(dwords >= 1 << 31, dwords - (1 << 32), dwords).to(torch.int32)
    return dwords.contiguous().view(torch.uint8).view(-1), sc.permute(0, 2, 3, 1, 4).contiguous().view(-1)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rand = lambda *shape: torch.randn(*shape, device=DEV, generator=g)  # noqa: E731
    if c["kind"] == "proj":
        rows = c["n"] * (2 if c["act"] == "swiglu" else 1)
        codes, scales = _pack_weights(c, (rand(rows, c["k"]) * 0.02).to(torch.bfloat16).float())
        st = dict(case=c, codes=codes, scales=scales, x=rand(c["m"], c["k"]).to(torch.bfloat16),
                  out=torch.zeros(c["m"], c["n"], dtype=torch.bfloat16, device=DEV), gain=None, resid=None)
        if c["norm"]:
            st["gain"] = (1 + 0.02 * rand(c["k"])).to(torch.bfloat16)
        if c["resid"]:
            st["resid"] = rand(c["m"], c["n"]).to(torch.bfloat16)
        return st
    B, KV, dh = c["n_seq"], c["kv_heads"], c["dh"]
    if c["kind"] == "evict":
        held = _lengths(c)
        codes, scales = _new_cache(dict(c, s_max=c["length"]), held, g)
        # few positions draw most of the weight, and some none at all
        u = torch.rand(B, KV, c["length"], device=DEV, generator=g)
        sums = torch.where(u < 0.1, torch.zeros_like(u), torch.exp(4 * u * rand(B, KV, c["length"])))
        s8 = _s8(c["keep"])
        return dict(case=c, codes=codes, scales=scales, sums=sums,
                    at=torch.tensor(held, dtype=torch.int32, device=DEV),
                    to_codes=torch.zeros(B * KV * s8 * dh, dtype=torch.uint8, device=DEV),
                    to_scales=torch.zeros(B, KV, 2, s8, dh // 32, dtype=torch.uint8, device=DEV),
                    to_sums=torch.zeros(B, KV, c["keep"], device=DEV),
                    idx=torch.zeros(B, KV, c["keep"], dtype=torch.int32, device=DEV),
                    kept=torch.tensor([min(n, c["keep"]) for n in held], dtype=torch.int32, device=DEV),
                    out=torch.zeros(B, c["keep"], 2 * KV * dh, dtype=torch.bfloat16, device=DEV))
    # the rows that a QKV projection of N(0, 0.02) weights gives from unit-RMS rows of d = 2048
    qkv = (rand(B * c["n_new"], (c["heads"] + 2 * KV) * dh) * 0.9).to(torch.bfloat16)
    held = [max(p, 0) + (0 if c["kind"] == "store" or p < 0 else c["n_new"]) for p in _positions(c)]
    codes, scales = _new_cache(c, held, g)
    at = torch.tensor(_positions(c), dtype=torch.int32, device=DEV)
    st = dict(case=c, qkv=qkv, codes=codes, scales=scales, at=at)
    if c["kind"] == "attn":
        st["out"] = torch.zeros(B * c["n_new"], c["heads"] * dh, dtype=torch.bfloat16, device=DEV)
        if c["sums"]:
            st["before"] = torch.rand(B, KV, c["s_max"], device=DEV, generator=g) * 4
            st["sums"] = torch.zeros_like(st["before"])
    else:
        st["lo"], st["hi"] = _window(c)
        # positions behind which a sequence has nothing to read back
        st["end"] = torch.where(at < 0, torch.zeros_like(at), at + c["n_new"])
        st["out"] = torch.zeros(B, st["hi"] - st["lo"], 2 * KV * dh, dtype=torch.bfloat16, device=DEV)
    return st


# -------------------------------------------------------------- plain forms

def _plain_weights(c, st, dtype=torch.float32):
    """The weights' values [rows, K]."""
    rows = c["n"] * (2 if c["act"] == "swiglu" else 1)
    T, C = -(-rows // 8), -(-c["k"] // 256)
    d = st["codes"].view(torch.int32).view(T, C, 4, 2, 8, 4).to(torch.int64) & 0xffffffff
    sc = st["scales"].view(T, C, 2, 8, 128 // c["group"])
    if c["fmt"] == "e2m1":
        code = (d[..., None] >> torch.arange(0, 32, 4, device=DEV)) & 15
        sc = torch.ldexp(torch.ones_like(sc, dtype=dtype), sc.int() - 127)
        v = _from_e2m1(code, dtype)
    else:
        i = torch.arange(4, device=DEV)
        mag = (d[..., None] >> torch.cat((8 * i, 8 * i + 4))) & 7
        neg = (d[..., None] >> torch.cat((8 * i + 7, (8 * i + 11) % 32))) & 1
        v, sc = torch.where(neg == 1, -mag, mag).to(dtype), sc.to(dtype)
    # t, c, g, h, r, s, e -> t, r, c, h, s, g, e
    v = v.permute(0, 4, 1, 3, 5, 2, 6).reshape(T, 8, C, 2, -1, c["group"])
    v = v * sc.permute(0, 3, 1, 2, 4)[..., None]
    return v.reshape(8 * T, 256 * C)[:rows, :c["k"]]


def _plain_proj(st):
    c = st["case"]
    x = st["x"].float()
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * st["gain"].float()
    y = torch.matmul(x, _plain_weights(c, st).t())
    if c["act"] == "swiglu":
        u, v = y[:, :c["n"]], y[:, c["n"]:]
        y = u / (1 + torch.exp(-u)) * v
    elif c["act"] == "relu2":
        y = y.clamp(min=0) ** 2
    if c["resid"]:
        y = y + st["resid"].float()
    return y.to(torch.bfloat16)


def _read(c, codes, scales, lo, hi):
    """Values of positions lo..hi-1 in float32, [n_seq, kv_heads, 2, hi - lo, dh]."""
    B, KV, dh = c["n_seq"], c["kv_heads"], c["dh"]
    t0, t1 = lo // 8, -(-hi // 8)
    k = _keys(c, codes)[:, :, lo:hi]
    k = torch.stack((k & 15, k >> 4), -1).flatten(-2)
    v = _values(c, codes)[:, :, t0:t1].permute(0, 1, 2, 5, 4, 3)        # tile, position, j, n
    v = torch.stack((v & 15, v >> 4), -2).reshape(B, KV, (t1 - t0) * 8, dh)[:, :, lo - 8 * t0:hi - 8 * t0]
    sc = scales[:, :, :, lo:hi]
    sc = torch.ldexp(torch.ones_like(sc, dtype=torch.float32), sc.int() - 127)
    x = _from_e2m1(torch.stack((k, v), 2))
    return (x.view(B, KV, 2, hi - lo, dh // 32, 32) * sc[..., None]).view(B, KV, 2, hi - lo, dh)


def _rows(x, end, lo):
    """Values [n_seq, kv_heads, 2, n, dh] as rows, those at or behind `end` as zeros."""
    B, n = x.shape[0], x.shape[3]
    x = x.permute(0, 3, 2, 1, 4).reshape(B, n, -1)
    left = torch.arange(lo, lo + n, device=DEV) < end[:, None]
    return torch.where(left[..., None], x, torch.zeros_like(x)).to(torch.bfloat16)


def _plain_store(st):
    c, codes, scales, at = st["case"], st["codes"], st["scales"], st["at"].long()
    B, H, KV, dh, n = c["n_seq"], c["heads"], c["kv_heads"], c["dh"], c["n_new"]
    lo, hi = st["lo"] // 8 * 8, _s8(st["hi"])
    p = torch.arange(lo, hi, device=DEV)
    new = (p >= at[:, None]) & (p < at[:, None] + n) & (at[:, None] >= 0)             # [B, window]
    rows = st["qkv"].view(B, n, H + 2 * KV, dh)[:, :, H:].float()
    code, sc = _quantise(rows.view(B, n, 2, KV, dh).permute(0, 3, 2, 1, 4).contiguous())
    j = (p - at[:, None]).clamp(0, n - 1)[:, None, None, :, None]
    code = torch.gather(code, 3, j.expand(B, KV, 2, -1, dh))
    sc = torch.gather(sc, 3, j.expand(B, KV, 2, -1, dh // 32))
    scales[:, :, :, lo:hi] = torch.where(new[:, None, None, :, None], sc, scales[:, :, :, lo:hi])
    k, v = _keys(c, codes)[:, :, lo:hi], _values(c, codes)[:, :, lo // 8:hi // 8]
    k.copy_(torch.where(new[:, None, :, None], _put_keys(code[:, :, 0]), k))
    v.copy_(torch.where(new.view(B, 1, -1, 1, 1, 8), _put_values(code[:, :, 1].contiguous()), v))
    return _rows(_read(c, codes, scales, st["lo"], st["hi"]), st["end"], st["lo"])


def _slopes(heads):
    n = 1 << (heads.bit_length() - 1)
    e = [-8 * (h + 1) / n if h < n else -4 * (2 * (h - n) + 1) / n for h in range(heads)]
    return torch.tensor([2.0 ** v for v in e], device=DEV)


def _plain_attn(st):
    c, at = st["case"], st["at"]
    B, H, KV, dh, n = c["n_seq"], c["heads"], c["kv_heads"], c["dh"], c["n_new"]
    G, S = H // KV, c["pos"] + n
    kv = _read(c, st["codes"], st["scales"], 0, S)
    q = st["qkv"].view(B, n, H + 2 * KV, dh)[:, :, :H].float().view(B, n, KV, G, dh).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q.reshape(B, KV, G * n, dh), kv[:, :, 0].transpose(-1, -2)).view(B, KV, G, n, S) / math.sqrt(dh)
    qp = at[:, None] + torch.arange(n, device=DEV)                                     # [B, n]
    back = qp[..., None] - torch.arange(S, device=DEV)                                 # [B, n, S]
    if c["alibi"]:
        s = s - _slopes(H).view(1, KV, G, 1, 1) * back[:, None, None].float()
    seen = ((back >= 0) & (at[:, None, None] >= 0))[:, None, None]
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    l = p.sum(-1, keepdim=True)
    p = (p / torch.where(l > 0, l, torch.ones_like(l))).view(B, KV, G * n, S)
    o = torch.matmul(p, kv[:, :, 1]).view(B, KV, G, n, dh).permute(0, 3, 1, 2, 4).reshape(B * n, H * dh)
    o = o.to(torch.bfloat16)
    if not c["sums"]:
        return o
    sums = st["before"].clone()
    sums[:, :, :S] += p.sum(2)
    return o, sums


def _plain_evict(st):
    c, at = st["case"], st["at"].long()
    B, KV, dh, S, keep, recent = c["n_seq"], c["kv_heads"], c["dh"], c["length"], c["keep"], c["recent"]
    p = torch.arange(S, device=DEV)
    held = (p < at[:, None])[:, None]
    # the last ones first of all, positions behind the last never
    last = (p >= (at - recent)[:, None])[:, None]
    rank = torch.where(held, torch.where(last, torch.full_like(st["sums"], math.inf), st["sums"]),
                       torch.full_like(st["sums"], -1.0))
    order = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :keep]
    order = torch.where(order < at[:, None, None], order, torch.full_like(order, S))
    idx = torch.sort(order, dim=-1)[0]
    idx = torch.nn.functional.pad(idx, (0, keep - idx.shape[-1]), value=S)
    there = idx < S
    i = torch.where(there, idx, torch.zeros_like(idx))
    x = _read(dict(c, s_max=S), st["codes"], st["scales"], 0, S)
    x = torch.gather(x, 3, i[:, :, None, :, None].expand(B, KV, 2, keep, dh))
    sums = torch.where(there, torch.gather(st["sums"], 2, i), torch.zeros_like(st["to_sums"]))
    idx = torch.where(there, idx, torch.full_like(idx, -1)).to(torch.int32)
    return idx, sums, _rows(x, st["kept"].long(), 0)


# ---------------------------------------------------- the framework's calls

def _handle(st):
    """Descriptors and workspace, made once as a program does."""
    if "ld" not in st:
        import paper_2609_05275_amd as ld
        c = st["case"]
        st["ld"], size = ld, 0
        if c["kind"] == "proj":
            rows = c["n"] * (2 if c["act"] == "swiglu" else 1)
            st["w"] = ld.w4(st["codes"], st["scales"], ld.LD_W4_E2M1 if c["fmt"] == "e2m1" else ld.LD_W4_INT4,
                            c["group"], rows, c["k"])
            st["act"] = {"none": ld.DEC_ACT_NONE, "swiglu": ld.DEC_ACT_SWIGLU, "relu2": ld.DEC_ACT_RELU2}[c["act"]]
            size = ld.ld_gemm_w4_ws_bytes(st["w"], c["m"], st["act"])
        elif c["kind"] == "evict":
            shape = (c["n_seq"], c["kv_heads"], c["dh"])
            st["kv"] = ld.kv4(st["codes"], st["scales"], *shape, c["length"], sums=st["sums"])
            st["to"] = ld.kv4(st["to_codes"], st["to_scales"], *shape, c["keep"], sums=st["to_sums"])
            size = ld.ld_kv4_evict_ws_bytes(st["kv"], c["length"], c["keep"])
        else:
            st["kv"] = ld.kv4(st["codes"], st["scales"], c["n_seq"], c["kv_heads"], c["dh"], c["s_max"],
                              sums=st.get("sums"))
            st["seq_pos"] = st["at"] if c["ragged"] else None
            if c["kind"] == "attn":
                size = ld.ld_attn_decode_kv4_ws_bytes(st["kv"], c["heads"], c["n_new"])
        st["ws"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    return st["ld"], st["case"]


def _own(st):
    ld, c = _handle(st)
    if c["kind"] == "proj":
        ld.ld_gemm_w4(st["w"], st["x"], st["out"], st["ws"], g=st["gain"], eps=EPS, R=st["resid"], act=st["act"])
        return st["out"]
    if c["kind"] == "attn":
        if c["sums"]:
            st["sums"].copy_(st["before"])
        ld.ld_attn_decode_kv4(st["kv"], c["heads"], c["pos"], c["n_new"], st["qkv"], st["out"], st["ws"],
                              seq_pos=st["seq_pos"], alibi=int(c["alibi"]))
        return (st["out"], st["sums"]) if c["sums"] else st["out"]
    if c["kind"] == "evict":
        ld.ld_kv4_evict(st["kv"], st["to"], c["length"], c["keep"], c["recent"], st["idx"], st["ws"],
                        seq_len=st["at"] if c["ragged"] else None)
        ld.ld_kv4_load(st["to"], 0, c["keep"], st["out"], seq_len=st["kept"] if c["ragged"] else None)
        return st["idx"], st["to_sums"], st["out"]
    ld.ld_kv4_store(st["kv"], c["heads"], c["n_new"], c["pos"], st["qkv"], seq_pos=st["seq_pos"])
    ld.ld_kv4_load(st["kv"], st["lo"], st["hi"] - st["lo"], st["out"], seq_len=st["end"] if c["ragged"] else None)
    return st["out"]


def run(state):
    if own:
        return _own(state)
    return {"proj": _plain_proj, "store": _plain_store, "attn": _plain_attn, "evict": _plain_evict}[state["case"]["kind"]](state)


# ------------------------------------------------------------- in 64 bits

def _value64(code):
    """What e2m1 codes stand for: 2 bits of exponent, 1 of mantissa."""
    e, m = (code >> 1) & 3, (code & 1).double()
    v = torch.where(e > 0, (2 + m) * torch.exp2(e.double() - 2), m / 2)
    return torch.where(code >= 8, -v, v)


def _round64(y):
    """y rounded to the nearest e2m1 value, ties to even, in float64."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)
    return torch.round(y / step) * step


def _exact_cache(c, codes, scales, b, h, part, count):
    """Values of the first `count` positions of one head, float64 [count, dh]."""
    dh = c["dh"]
    s8 = scales.shape[3]
    at = ((b * c["kv_heads"] + h) * 2 + part) * s8 * (dh // 2)
    raw = codes[at:at + s8 * (dh // 2)].to(torch.int64)
    if part == 0:
        raw = raw.view(s8, dh // 2)
        code = torch.zeros(s8, dh, dtype=torch.int64, device=DEV)
        code[:, 0::2], code[:, 1::2] = raw & 15, raw >> 4
    else:
        raw = raw.view(s8 // 8, 16, dh // 32, 8)
        code = torch.zeros(s8 // 8, 8, dh // 32, 32, dtype=torch.int64, device=DEV)
        for n in range(16):
            code[..., n] = (raw[:, n] & 15).transpose(1, 2)
            code[..., 16 + n] = (raw[:, n] >> 4).transpose(1, 2)
        code = code.view(s8, dh)
    s = torch.exp2(scales[b, h, part].double() - 127).repeat_interleave(32, -1)
    return (_value64(code) * s)[:count]


def _exact_proj(c, st):
    x = st["x"].double()
    if c["norm"]:
        x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + EPS) * st["gain"].double()
    rows = c["n"] * (2 if c["act"] == "swiglu" else 1)
    K, C = c["k"], -(-c["k"] // 256)
    raw = st["codes"].view(torch.int32).to(torch.int64) & 0xffffffff
    y = torch.zeros(c["m"], rows, dtype=torch.float64, device=DEV)
    k = torch.arange(K, device=DEV)
    lane, dword, e = 16 * (k // 8 % 4) + 8 * (k // 128 % 2), k // 32 % 4, k % 8
    for n0 in range(0, rows, 4096):
        n = torch.arange(n0, min(rows, n0 + 4096), device=DEV)[:, None]
        d = raw[(((n // 8) * C + k // 256) * 64 + lane + n % 8) * 4 + dword]
        per = 128 // c["group"]
        s = st["scales"][((((n // 8) * C + k // 256) * 2 + k // 128 % 2) * 8 + n % 8) * per + k % 128 // c["group"]]
        if c["fmt"] == "e2m1":
            w = _value64((d >> (4 * e)) & 15) * torch.exp2(s.double() - 127)
        else:
            mag = (d >> (8 * (e % 4) + 4 * (e // 4))) & 7
            neg = (d >> ((8 * (e % 4) + 7 + 4 * (e // 4)) % 32)) & 1
            w = (mag * (1 - 2 * neg)).double() * s.double()
        y[:, n0:n0 + 4096] = x @ w.t()
    if c["act"] == "swiglu":
        y = y[:, :c["n"]] * torch.sigmoid(y[:, :c["n"]]) * y[:, c["n"]:]
    elif c["act"] == "relu2":
        y = torch.relu(y).square()
    return y + st["resid"].double() if c["resid"] else y


def _exact_attn(c, st):
    B, H, KV, dh, n = c["n_seq"], c["heads"], c["kv_heads"], c["dh"], c["n_new"]
    rows = st["qkv"].double().view(B, n, H + 2 * KV, dh)
    out = torch.zeros(B, n, H, dh, dtype=torch.float64, device=DEV)
    sums = st["before"].double() if c["sums"] else None
    slopes = _slopes(H).double()
    for b, pos in enumerate(_positions(c)):
        if pos < 0:
            continue
        keys = torch.arange(pos + n, device=DEV)
        for h in range(H):
            kvh = h // (H // KV)
            if h % (H // KV) == 0:
                k, v = (_exact_cache(c, st["codes"], st["scales"], b, kvh, part, pos + n) for part in (0, 1))
            for j in range(n):
                s = (k @ rows[b, j, h]) / math.sqrt(dh)
                if c["alibi"]:
                    s = s - slopes[h] * (pos + j - keys)
                w = torch.softmax(s[:pos + j + 1], 0)
                out[b, j, h] = w @ v[:pos + j + 1]
                if sums is not None:
                    sums[b, kvh, :pos + j + 1] += w
    out = out.view(B * n, H * dh)
    return out if sums is None else (out, sums)


def _exact_evict(c, st):
    B, KV, dh, keep, recent = c["n_seq"], c["kv_heads"], c["dh"], c["keep"], c["recent"]
    sums = torch.zeros(B, KV, keep, dtype=torch.float64, device=DEV)
    out = torch.zeros(B, keep, 2, KV, dh, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(c)):
        for h in range(KV):
            w = st["sums"][b, h, :n].double()
            if n <= keep:
                at = torch.arange(n, device=DEV)
            else:
                old = w[:n - recent]
                # the smallest of those kept, and of its equals the first ones
                least = torch.topk(old, keep - recent)[0][-1] if keep > recent else math.inf
                more, same = torch.nonzero(old > least)[:, 0], torch.nonzero(old == least)[:, 0]
                at = torch.cat((more, same[:keep - recent - len(more)])).sort()[0]
                at = torch.cat((at, torch.arange(n - recent, n, device=DEV)))
            sums[b, h, :len(at)] = w[at]
            for part in (0, 1):
                out[b, :len(at), part, h] = _exact_cache(c, st["codes"], st["scales"], b, h, part, n)[at]
    return None, sums, out.view(B, keep, 2 * KV * dh)


def _exact_store(c, st):
    B, H, KV, dh, n = c["n_seq"], c["heads"], c["kv_heads"], c["dh"], c["n_new"]
    lo, hi = st["lo"], st["hi"]
    rows = st["qkv"].double().view(B, n, H + 2 * KV, dh)
    out = torch.zeros(B, hi - lo, 2, KV, dh, dtype=torch.float64, device=DEV)
    for b, pos in enumerate(_positions(c)):
        if pos < 0:
            continue
        for h in range(KV):
            for part in (0, 1):
                x = rows[b, :, H + part * KV + h].reshape(n, dh // 32, 32)
                e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 6)).clamp(min=MIN_EXP)
                x = (_round64(x / torch.exp2(e)) * torch.exp2(e)).view(n, dh)
                was = _exact_cache(c, st["codes"], st["scales"], b, h, part, pos)
                out[b, :pos + n - lo, part, h] = torch.cat((was, x))[lo:]
    return out.view(B, hi - lo, 2 * KV * dh)


def exact(case, seed):
    st = prepare(case, seed)
    return {"proj": _exact_proj, "store": _exact_store, "attn": _exact_attn, "evict": _exact_evict}[case["kind"]](case, st)
