"""The 8-bit key/value cache and its attention, as measurable cases.

Three operators, reached through the package's entry points:

  store   ld_kv8_store of the key/value columns of new rows, and ld_kv8_load
          of the rows of the blocks it touched: the values the cache then
          stands for (a prompt, or a few rows appended to a longer cache)
  load    ld_kv8_load: codes and scales back to bfloat16 rows
  attn    ld_attn_decode_kv8: queries of 1 to 8 new rows per sequence over the
          cache (one row: a token of plain decoding; several: the verify step
          of speculative decoding)

The cache of one (sequence, key/value head) is its keys [S16][dh] in bytes,
then its values [S16 / 16][dh][16], S16 being the positions rounded up to 16.
A scale, a power of two in float32, belongs to a block of positions of one
head's keys or values: scales [n_seq][kv_heads][2][blocks].  With Q = 448
(e4m3) or 127 (int8), a block needs the smallest 2^e (e >= -100) with
max|x| <= Q 2^e; a block that the call starts takes what its new rows need, one
that holds earlier rows the larger of that and its old scale, earlier codes
being rounded again when it grows.  A code is x / scale rounded to nearest even.

Ragged cases give each sequence its own position, and leave every fifth out.
"""
import math

import torch

own = False

DEV = "cuda:0"
QMAX = {"e4m3": 448.0, "int8": 127.0}
MIN_EXP = -100


# ------------------------------------------------------------------- cases

def _case(name, kind, fmt, block, n_seq, heads, kv_heads, dh, s_max, pos, n_new, ragged=0, alibi=False):
    return dict(name=name, kind=kind, fmt=fmt, block=block, n_seq=n_seq, heads=heads, kv_heads=kv_heads, dh=dh,
                s_max=s_max, pos=pos, n_new=n_new, ragged=ragged, alibi=alibi)


def listed():
    return [
        # one token of one sequence of the 125M shape into a part-filled block:
        # launches and host time are everything
        _case("append_125m_b1", "store", "int8", 32, 1, 12, 12, 64, 1024, 777, 1),
        # a decoding step's token for 32 sequences of the 1B shape, each at
        # its own position
        _case("append_1b_b32", "store", "e4m3", 64, 32, 16, 16, 128, 2056, 2047, 1, ragged=90),
        # the prompts of the 1B shape at its training length
        _case("prompt_1b_b8", "store", "e4m3", 64, 8, 16, 16, 128, 2112, 0, 2048),
        # prompts of odd length, four query heads to a key/value head, the
        # smallest blocks
        _case("prompt_gqa_b3", "store", "int8", 16, 3, 32, 8, 128, 1504, 0, 1501),
        # a window in the middle of a short cache (an earlier turn's
        # rows, wanted in bfloat16)
        _case("load_125m_window", "load", "int8", 128, 1, 12, 12, 64, 1024, 333, 100),
        # whole caches of the 7B shape back to bfloat16
        _case("load_7b", "load", "e4m3", 64, 4, 32, 32, 128, 4096, 0, 4096),
        # a token over a short cache, the smallest attention
        _case("attn_125m_b1", "attn", "int8", 32, 1, 12, 12, 64, 1024, 199, 1),
        # interactive decoding of the 1B shape
        _case("attn_1b_b1", "attn", "e4m3", 64, 1, 16, 16, 128, 1024, 777, 1),
        # the verify step after a draft of five
        _case("verify_1b_b8", "attn", "int8", 32, 8, 16, 16, 128, 1536, 1500, 6),
        # the paper's own block (ALiBi): a token of eight sequences
        _case("attn_3p9b_b8", "attn", "int8", 64, 8, 16, 16, 128, 4096, 4000, 1, alibi=True),
        # two long contexts, four query heads to a key/value head: little to
        # spread over the chip but the cache's length
        _case("attn_gqa_long", "attn", "e4m3", 128, 2, 32, 8, 128, 131072, 131071, 1),
        # a serving batch of the 7B shape, lengths from none to 8192
        _case("attn_7b_b16", "attn", "e4m3", 64, 16, 32, 32, 128, 8192, 8191, 1, ragged=8191),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same kinds and ranges."""
    kind = rng.choice(["store", "prompt", "load", "attn", "attn", "attn"])
    dh = rng.choice([64, 128, 128])
    kv_heads = rng.choice([4, 8, 12, 16, 20, 32])
    group = rng.choice([1, 1, 1, 2, 4, 8])
    n_seq = _log_int(rng, 1, 32)
    fmt, block = rng.choice(["e4m3", "int8"]), rng.choice([16, 32, 64, 128])
    if kind == "prompt":
        n_new, pos, ragged = _log_int(rng, 20, 4000), rng.choice([0, 0, _log_int(rng, 1, 500)]), 0
        # no more rows than the largest listed prompts
        most = 8 * 2048 * 16 * 128
    elif kind == "store":
        n_new, pos = rng.randint(1, 8), _log_int(rng, 1, 8000)
        ragged, most = rng.choice([0, min(pos, 2 * block)]), None
    elif kind == "load":
        n_new, pos, ragged = _log_int(rng, 20, 4096), rng.choice([0, _log_int(rng, 1, 1000)]), 0
        most = 4 * 4096 * 32 * 128
    else:
        n_new, pos = rng.choice([1, 1, rng.randint(2, 8)]), _log_int(rng, 30, 100000)
        ragged, most = rng.choice([0, 0, pos]), None
    rows = n_new if most else pos + n_new
    most = most or 2 * 131072 * 8 * 128 // max(1, n_new * group // 16)
    while n_seq > 1 and n_seq * rows * kv_heads * dh > most:
        n_seq //= 2
    while rows * kv_heads * dh > most and kv_heads > 4:
        kv_heads //= 2
    c = _case("", "store" if kind == "prompt" else kind, fmt, block, n_seq, group * kv_heads, kv_heads, dh,
              pos + n_new + rng.randint(0, 200), pos, n_new, ragged, kind == "attn" and rng.random() < 0.3)
    del c["name"]
    return c


# ------------------------------------------------------------ shared sizes

def _positions(c):
    """Each sequence's first new position: pos, or for ragged cases spread
    over the `ragged` positions before it, with every fifth sequence left out."""
    if not c["ragged"]:
        return [c["pos"]] * c["n_seq"]
    return [-1 if b % 5 == 4 else c["pos"] - (b * 7919) % (c["ragged"] + 1) for b in range(c["n_seq"])]


def _window(c):
    """First and last + 1 position that a store case reads back: from the
    start of the first block it may touch."""
    lo = min(p for p in _positions(c) if p >= 0)
    return lo - lo % c["block"], c["pos"] + c["n_new"]


def work(case):
    c = case
    d = c["kv_heads"] * c["dh"]
    at = [p for p in _positions(c) if p >= 0]
    if c["kind"] == "store":
        # new rows in, their codes out, the other rows' codes in, all rows out in bfloat16
        w0 = _window(c)[0]
        old = sum(p - max(w0, 0) for p in at)
        new = len(at) * c["n_new"]
        return dict(bytes=2 * d * (2 * new + new + old + 2 * (new + old)), flops=0)
    if c["kind"] == "load":
        return dict(bytes=2 * d * 3 * c["n_seq"] * c["n_new"], flops=0)
    keys = sum(p + c["n_new"] for p in at)
    pairs = sum(c["n_new"] * (p + (c["n_new"] + 1) / 2) for p in at)
    rows = c["n_seq"] * c["n_new"] * c["heads"] * c["dh"]
    return dict(bytes=2 * d * keys + 8 * c["kv_heads"] * keys / c["block"] + 2 * rows * 2,
                flops=4 * c["heads"] * c["dh"] * pairs)


# ------------------------------------------------------------------ inputs

def _s16(c):
    return (c["s_max"] + 15) // 16 * 16


def _keys(c, codes):
    """Keys of all positions, [n_seq, kv_heads, S16, dh], as a view of the codes."""
    return codes.view(c["n_seq"], c["kv_heads"], 2, _s16(c), c["dh"])[:, :, 0]


def _values(c, codes):
    """Values of all positions, [n_seq, kv_heads, S16 / 16, dh, 16], as a view."""
    return codes.view(c["n_seq"], c["kv_heads"], 2, _s16(c) // 16, c["dh"], 16)[:, :, 1]


def _as_float(c, codes):
    return codes.view(torch.float8_e4m3fn if c["fmt"] == "e4m3" else torch.int8).float()


def _to_code(c, x):
    """Codes (as bytes) of values already divided by their scale."""
    if c["fmt"] == "e4m3":
        return x.to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.round(x).to(torch.int8).view(torch.uint8)


def _need(c, amax):
    """Smallest 2^e, e >= MIN_EXP, with amax <= Q 2^e, in float32."""
    m, e = torch.frexp(amax)                      # amax = m 2^e, m in [1/2, 1)
    qm, qe = math.frexp(QMAX[c["fmt"]])
    e = torch.where(m > qm, e + 1, e) - qe
    e = torch.where(amax > 0, e, torch.full_like(e, MIN_EXP)).clamp(min=MIN_EXP)
    return torch.ldexp(torch.ones_like(amax), e)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    B, H, KV, dh, blk = c["n_seq"], c["heads"], c["kv_heads"], c["dh"], c["block"]
    s16, nb = _s16(c), -(-c["s_max"] // c["block"])
    # the rows that a QKV projection of N(0, 0.02) weights gives from unit-RMS
    # rows of d = 2048
    qkv = (torch.randn(B * c["n_new"], (H + 2 * KV) * dh, device=DEV, generator=g) * 0.9).to(torch.bfloat16)
    codes = torch.zeros(B * KV * 2 * s16 * dh, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(B, KV, 2, nb, device=DEV)
    held = [max(p, 0) + (0 if c["kind"] == "store" else c["n_new"]) for p in _positions(c)]  # filled positions
    step = max(blk, (1 << 24) // (KV * dh) // blk * blk)  # blocks, a piece at a time
    for b in range(B):
        for p0 in range(0, held[b], step):
            n = min(step, s16 - p0)
            x = torch.randn(KV, 2, n, dh, device=DEV, generator=g) * 0.9
            x = x.to(torch.bfloat16).float()
            x[:, :, max(held[b] - p0, 0):] = 0
            x = torch.nn.functional.pad(x, (0, 0, 0, -n % blk)).view(KV, 2, -1, blk, dh)
            sc = _need(c, x.abs().amax((-1, -2)))
            q = _to_code(c, x / sc[..., None, None]).view(KV, 2, -1, dh)[:, :, :n]
            scales[b, :, :, p0 // blk: p0 // blk + min(sc.shape[2], nb - p0 // blk)] = sc[:, :, :nb - p0 // blk]
            _keys(c, codes)[b, :, p0:p0 + n] = q[:, 0]
            _values(c, codes)[b, :, p0 // 16:(p0 + n) // 16] = q[:, 1].reshape(KV, n // 16, 16, dh).transpose(-1, -2)
    at = torch.tensor(_positions(c), dtype=torch.int32, device=DEV)
    st = dict(case=c, qkv=qkv, codes=codes, scales=scales, at=at)
    if c["kind"] == "attn":
        st["out"] = torch.zeros(B * c["n_new"], H * dh, dtype=torch.bfloat16, device=DEV)
    else:
        lo, hi = _window(c) if c["kind"] == "store" else (c["pos"], c["pos"] + c["n_new"])
        st["lo"], st["hi"] = lo, hi
        # positions behind which a sequence has nothing to read back
        st["end"] = torch.where(at < 0, torch.zeros_like(at), at + c["n_new"])
        st["out"] = torch.zeros(B, hi - lo, 2 * KV * dh, dtype=torch.bfloat16, device=DEV)
    return st


# -------------------------------------------------------------- plain forms

def _read(c, codes, scales, lo, hi):
    """Values of positions lo..hi-1 in float32, [n_seq, kv_heads, 2, hi - lo, dh]."""
    B, KV, dh = c["n_seq"], c["kv_heads"], c["dh"]
    t0, t1 = lo // 16, -(-hi // 16)
    k = _as_float(c, _keys(c, codes)[:, :, lo:hi].contiguous())
    v = _values(c, codes)[:, :, t0:t1].transpose(-1, -2).contiguous().view(B, KV, (t1 - t0) * 16, dh)
    v = _as_float(c, v[:, :, lo - 16 * t0:hi - 16 * t0].contiguous())
    sc = scales[..., torch.arange(lo, hi, device=DEV) // c["block"]]
    return torch.stack((k, v), 2) * sc[..., None]


def _plain_store(st):
    c, codes, scales, at = st["case"], st["codes"], st["scales"], st["at"].long()
    B, H, KV, dh, blk, n = c["n_seq"], c["heads"], c["kv_heads"], c["dh"], c["block"], c["n_new"]
    lo = st["lo"]
    hi = min(-(-st["hi"] // blk) * blk, _s16(c))
    W, nb = hi - lo, -(-(hi - lo) // blk)
    p = torch.arange(lo, lo + nb * blk, device=DEV)
    new = (p >= at[:, None]) & (p < at[:, None] + n) & (at[:, None] >= 0)             # [B, window]
    rows = st["qkv"].view(B, n, H + 2 * KV, dh)[:, :, H:].float()
    rows = rows.view(B, n, 2, KV, dh).permute(0, 3, 2, 1, 4)                          # [B, KV, 2, n, dh]
    j = (p - at[:, None]).clamp(0, n - 1)
    x = torch.gather(rows, 3, j[:, None, None, :, None].expand(B, KV, 2, -1, dh))
    x = torch.where(new[:, None, None, :, None], x, torch.zeros_like(x)).view(B, KV, 2, nb, blk, dh)
    s0 = scales[..., lo // blk:lo // blk + nb]
    need = _need(c, x.abs().amax((-1, -2)))
    touched = new.view(B, nb, blk).any(-1)[:, None, None]
    goes_on = (p.view(nb, blk)[:, 0] < at[:, None])[:, None, None]
    s1 = torch.where(touched, torch.where(goes_on, torch.maximum(need, s0), need), s0)
    was = torch.nn.functional.pad(_read(c, codes, scales, lo, hi), (0, 0, 0, nb * blk - W)).view(B, KV, 2, nb, blk, dh)
    y = torch.where(new.view(B, 1, 1, nb, blk, 1), x, was)
    q = _to_code(c, y / torch.where(s1 > 0, s1, torch.ones_like(s1))[..., None, None]).view(B, KV, 2, nb * blk, dh)
    scales[..., lo // blk:lo // blk + nb] = s1
    _keys(c, codes)[:, :, lo:hi] = q[:, :, 0, :W]
    _values(c, codes)[:, :, lo // 16:hi // 16] = q[:, :, 1, :W].reshape(B, KV, W // 16, 16, dh).transpose(-1, -2)
    return _plain_load(st)


def _plain_load(st):
    c, lo, hi = st["case"], st["lo"], st["hi"]
    x = _read(c, st["codes"], st["scales"], lo, hi).permute(0, 3, 2, 1, 4).reshape(c["n_seq"], hi - lo, -1)
    left = torch.arange(lo, hi, device=DEV) < st["end"][:, None]
    return torch.where(left[..., None], x, torch.zeros_like(x)).to(torch.bfloat16)


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
    o = torch.matmul((p / torch.where(l > 0, l, torch.ones_like(l))).view(B, KV, G * n, S), kv[:, :, 1])
    return o.view(B, KV, G, n, dh).permute(0, 3, 1, 2, 4).reshape(B * n, H * dh).to(torch.bfloat16)


# ---------------------------------------------------- the framework's calls

def _handle(st):
    """The cache's descriptor and the workspace, made once as a program does."""
    if "kv" not in st:
        import paper_2609_05275_amd as ld
        c = st["case"]
        st["ld"] = ld
        st["kv"] = ld.kv8(st["codes"], st["scales"], ld.LD_KV8_E4M3 if c["fmt"] == "e4m3" else ld.LD_KV8_INT8,
                          c["block"], c["n_seq"], c["kv_heads"], c["dh"], c["s_max"])
        st["seq_pos"] = st["at"] if c["ragged"] else None
        st["seq_len"] = st["end"] if c["kind"] == "store" and c["ragged"] else None
        if c["kind"] == "attn":
            st["ws"] = torch.empty(ld.ld_attn_decode_kv8_ws_bytes(st["kv"], c["heads"], c["n_new"]),
                                   dtype=torch.uint8, device=DEV)
    return st["ld"], st["kv"], st["case"]


def _own(st):
    ld, kv, c = _handle(st)
    if c["kind"] == "attn":
        ld.ld_attn_decode_kv8(kv, c["heads"], c["pos"], c["n_new"], st["qkv"], st["out"], st["ws"],
                              seq_pos=st["seq_pos"], alibi=int(c["alibi"]))
        return st["out"]
    if c["kind"] == "store":
        ld.ld_kv8_store(kv, c["heads"], c["n_new"], c["pos"], st["qkv"], seq_pos=st["seq_pos"])
    ld.ld_kv8_load(kv, st["lo"], st["hi"] - st["lo"], st["out"], seq_len=st["seq_len"])
    return st["out"]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return _plain_store(state) if kind == "store" else _plain_load(state) if kind == "load" else _plain_attn(state)


# ------------------------------------------------------------- in 64 bits

def _round64(c, x):
    """x rounded to the format's nearest value, ties to even, in float64."""
    if c["fmt"] == "int8":
        return torch.round(x)
    # normal e4m3 steps are 2^(e - 3) for 2^e <= |x| < 2^(e + 1); 2^-9 below 2^-6
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_values(c, st, b, h, part, count):
    """Values of the first `count` positions of one head, float64 [count, dh]."""
    s16, dh = _s16(c), c["dh"]
    at = ((b * c["kv_heads"] + h) * 2 + part) * s16 * dh
    raw = st["codes"][at:at + s16 * dh]
    raw = raw.view(s16, dh) if part == 0 else raw.view(s16 // 16, dh, 16).permute(0, 2, 1).reshape(s16, dh)
    raw = raw[:count].contiguous().to(torch.int64)
    if c["fmt"] == "int8":
        val = (raw - 256 * (raw >= 128)).double()
    else:
        e, m = (raw >> 3) & 15, (raw & 7).double()
        val = torch.where(e > 0, (8 + m) * torch.exp2(e.double() - 10), m * 2.0 ** -9)
        val = torch.where(raw >= 128, -val, val)
    s = st["scales"][b, h, part].double().repeat_interleave(c["block"])[:count]
    return val * s[:, None]


def exact(case, seed):
    c = case
    B, H, KV, dh, blk, n = c["n_seq"], c["heads"], c["kv_heads"], c["dh"], c["block"], c["n_new"]
    st = prepare(c, seed)
    pos = _positions(c)
    rows = st["qkv"].double().view(B, n, H + 2 * KV, dh)
    if c["kind"] == "attn":
        out = torch.zeros(B, n, H, dh, dtype=torch.float64, device=DEV)
        slopes = _slopes(H).double()
        for b in range(B):
            if pos[b] < 0:
                continue
            keys = torch.arange(pos[b] + n, device=DEV)
            for h in range(H):
                if h % (H // KV) == 0:
                    k, v = (_exact_values(c, st, b, h // (H // KV), part, pos[b] + n) for part in (0, 1))
                for j in range(n):
                    s = (k @ rows[b, j, h]) / math.sqrt(dh)
                    if c["alibi"]:
                        s = s - slopes[h] * (pos[b] + j - keys)
                    w = torch.softmax(s[:pos[b] + j + 1], 0)
                    out[b, j, h] = w @ v[:pos[b] + j + 1]
        return out.view(B * n, H * dh)
    lo, hi = st["lo"], st["hi"]
    out = torch.zeros(B, hi - lo, 2, KV, dh, dtype=torch.float64, device=DEV)
    for b in range(B):
        if pos[b] < 0:
            continue
        for h in range(KV):
            for part in (0, 1):
                x = _exact_values(c, st, b, h, part, hi if c["kind"] == "load" else pos[b])
                if c["kind"] == "store":
                    new = rows[b, :, H + part * KV + h]
                    end = pos[b] + n
                    x = torch.cat((x, new))
                    # the blocks touched, padded to whole ones: what each needs
                    b0 = pos[b] // blk
                    y = torch.nn.functional.pad(new, (0, 0, pos[b] - b0 * blk, -end % blk)).view(-1, blk * dh)
                    e = torch.ceil(torch.log2(y.abs().amax(1) / QMAX[c["fmt"]])).clamp(min=MIN_EXP)
                    s = torch.exp2(e)
                    if pos[b] % blk:
                        s[0] = torch.maximum(s[0], st["scales"][b, h, part, b0].double())
                    s = s.repeat_interleave(blk)[:end - b0 * blk, None]
                    x[b0 * blk:] = _round64(c, x[b0 * blk:] / s) * s
                else:
                    end = hi
                out[b, :end - lo, part, h] = x[lo:end]
    return out.view(B, hi - lo, 2 * KV * dh)
