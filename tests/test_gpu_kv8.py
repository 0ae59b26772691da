"""The 8-bit key/value cache on the HIP path against the float64 oracle: codes
and scales bit for bit, values read back exactly, attention within a bound that
counts its roundings."""
import numpy as np
import pytest
import torch

import paper_2609_05275_amd as ld
from oracle import kv8
from tests.gpu_util import DEV, f64

pytestmark = pytest.mark.gpu

FMTS = pytest.mark.parametrize("fmt", [kv8.E4M3, kv8.INT8], ids=["e4m3", "int8"])
BLOCKS = pytest.mark.parametrize("block", [16, 32, 64, 128])
DHS = pytest.mark.parametrize("dh", [64, 128])
FILL = 0x7F     # NaN as e4m3: what memory that nobody wrote holds


class Dev:
    """A cache on the GPU whose memory held NaNs, and its oracle."""

    def __init__(self, fmt, block, n_seq, kv_heads, dh, s_max):
        self.ref = kv8.Cache(fmt, block, n_seq, kv_heads, dh, s_max)
        self.ref.scale[:] = np.nan
        self.ref.code[:] = np.nan if fmt == kv8.E4M3 else FILL
        self.shape = (n_seq, kv_heads, dh, s_max)
        self.fmt = ld.LD_KV8_E4M3 if fmt == kv8.E4M3 else ld.LD_KV8_INT8
        probe = ld.kv8(None, None, self.fmt, block, n_seq, kv_heads, dh, s_max)
        self.codes = torch.full((ld.ld_kv8_code_bytes(probe),), FILL, dtype=torch.uint8, device=DEV)
        self.scales = torch.full((ld.ld_kv8_scale_bytes(probe) // 4,), float("nan"), device=DEV)
        self.kv = ld.kv8(self.codes, self.scales, self.fmt, block, n_seq, kv_heads, dh, s_max)

    def upload(self):
        """The oracle's contents (finite where written) to the GPU."""
        code = np.where(np.isnan(self.ref.code), 0.0, self.ref.code)
        raw = np.where(np.isnan(self.ref.code), FILL, kv8.to_bytes(self.ref.fmt, code))
        keep, self.ref.code = self.ref.code, code
        packed = self.ref.pack(fill=FILL)
        self.ref.code = keep
        # bytes that were never written stay the fill
        mask = kv8.Cache(self.ref.fmt, 16, *self.ref.code.shape[:2], self.shape[2], self.shape[3])
        mask.fmt, mask.code = kv8.INT8, np.isnan(keep).astype(np.float64)
        packed = np.where(mask.pack() != 0, FILL, packed).astype(np.uint8)
        assert np.array_equal(kv8.unpack(packed, *self.shape[:2], *self.shape[2:]), raw)
        self.codes.copy_(torch.from_numpy(packed))
        self.scales.copy_(torch.from_numpy(self.ref.scale.reshape(-1)).float())

    def raw(self):
        n, kvh, dh, s_max = self.shape
        return kv8.unpack(self.codes.cpu().numpy(), n, kvh, dh, s_max), \
            f64(self.scales).reshape(self.ref.scale.shape)

    def store(self, x, pos, n_heads=None, seq_pos=False):
        """x [n_seq, n, 2, KV, dh] in bf16; pos: list, None for a sequence left out."""
        n_seq, n, _, kvh, dh = x.shape
        H = n_heads or kvh
        qkv = torch.randn(n_seq, n, (H + 2 * kvh) * dh).to(torch.bfloat16)
        qkv[:, :, H * dh:] = x.reshape(n_seq, n, -1)
        top = max(p for p in pos if p is not None)
        sp = torch.tensor([-1 if p is None else p for p in pos], dtype=torch.int32, device=DEV) if seq_pos else None
        ld.ld_kv8_store(self.kv, H, n, top, qkv.to(DEV).view(n_seq * n, -1), seq_pos=sp)
        self.ref.store(x.double().numpy(), pos)
        return qkv


def same(dev, length):
    """Codes of the positions below length[b] and the scales of their blocks."""
    code, scale = dev.raw()
    for b, n in enumerate(length):
        nb = -(-n // dev.ref.block)
        np.testing.assert_array_equal(scale[b, :, :, :nb], dev.ref.scale[b, :, :, :nb])
        bad = np.isnan(np.repeat(dev.ref.scale[b], dev.ref.block, -1)[..., :n])       # codes of NaN blocks say nothing
        want = kv8.to_bytes(dev.ref.fmt, dev.ref.code[b, :, :, :n])
        np.testing.assert_array_equal(np.where(bad[..., None], 0, code[b, :, :, :n]), np.where(bad[..., None], 0, want))
        # nothing is written behind the tile of 16 that holds the last position
        t = -(-n // 16) * 16
        assert np.all(code[b, :, :, t:] == FILL)
        assert np.all(np.isnan(scale[b, :, :, nb:]))


def rows(rng, *shape, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


# ---------------------------------------------------------------- store, load

@FMTS
@BLOCKS
@DHS
@pytest.mark.parametrize("n", [1, 15, 16, 64, 129, 200])
def test_store_prompt(fmt, block, dh, n):
    rng = np.random.default_rng(n + block)
    dev = Dev(fmt, block, 2, 3, dh, 203)
    x = rows(rng, 2, n, 2, 3, dh)
    x *= torch.from_numpy(2.0 ** rng.integers(-6, 7, (2, n, 2, 3, 1))).to(torch.bfloat16)   # rows of many sizes
    dev.store(x, [0, 0], n_heads=6)
    same(dev, [n, n])


@FMTS
@BLOCKS
@DHS
def test_store_appends(fmt, block, dh):
    """Rows one call after another, growing in size so that blocks are rounded
    again, into blocks begun before; then overwritten from the middle, as a
    verify step does."""
    rng = np.random.default_rng(7 * block + dh)
    dev = Dev(fmt, block, 2, 2, dh, 300)
    at = 0
    for i, n in enumerate([37, 1, 1, 8, 5, 1, 64, 3, 1, 100, 8]):
        dev.store(rows(rng, 2, n, 2, 2, dh, scale=1.5 ** i), [at, at])
        at += n
        same(dev, [at, at])
    at -= 8 + 50
    dev.store(rows(rng, 2, 6, 2, 2, dh, scale=300.0), [at, at])
    code, scale = dev.raw()
    np.testing.assert_array_equal(code[:, :, :, :at + 6], kv8.to_bytes(fmt, dev.ref.code[:, :, :, :at + 6]))
    nb = -(-(at + 6) // block)
    np.testing.assert_array_equal(scale[..., :nb], dev.ref.scale[..., :nb])


@FMTS
@BLOCKS
def test_store_ragged(fmt, block):
    """Each sequence at its own position, some left out; whatever is outside
    [0, pos] counts as left out."""
    rng = np.random.default_rng(block)
    dev = Dev(fmt, block, 6, 2, 64, 260)
    pos = [0, 17, None, 127, 128, None]
    dev.store(rows(rng, 6, 140, 2, 2, 64), [0] * 6)
    before = dev.raw()
    for n in (1, 8, 100):
        x = rows(rng, 6, n, 2, 2, 64, scale=n)
        sp = torch.tensor([0, 17, -5, 127, 128, 10 ** 9], dtype=torch.int32, device=DEV)
        qkv = x.reshape(6 * n, -1)
        qkv = torch.cat((torch.zeros(6 * n, 128, dtype=torch.bfloat16), qkv), 1).to(DEV)
        ld.ld_kv8_store(dev.kv, 2, n, 128, qkv, seq_pos=sp)
        dev.ref.store(x.double().numpy(), pos)
        code, scale = dev.raw()
        for b, p in enumerate(pos):
            if p is None:
                np.testing.assert_array_equal(code[b], before[0][b])
                np.testing.assert_array_equal(scale[b], before[1][b])
            else:
                nb = -(-(p + n) // block)
                np.testing.assert_array_equal(code[b, :, :, :p + n], kv8.to_bytes(fmt, dev.ref.code[b, :, :, :p + n]))
                np.testing.assert_array_equal(scale[b, :, :, :nb], dev.ref.scale[b, :, :, :nb])


@FMTS
def test_store_extreme_values(fmt):
    """Zeros, subnormals, the largest values, exact limits of a scale and the next
    value above, ties, infinities and NaNs."""
    q = kv8.QMAX[fmt]
    dev = Dev(fmt, 16, 1, 1, 64, 160)
    x = torch.zeros(1, 160, 2, 1, 64, dtype=torch.bfloat16)
    x[0, 16:32] = 2.0 ** -130
    x[0, 32:48] = torch.finfo(torch.bfloat16).max
    x[0, 48, :, 0, 3] = q * 2.0 ** -5
    x[0, 64, :, 0, 3] = torch.from_numpy(np.array(-q * 2.0 ** -5 * (1 + 2.0 ** -6))).to(torch.bfloat16)
    x[0, 49:64, :, 0, 5] = (torch.arange(15, dtype=torch.bfloat16) * 2.0 ** -6)[:, None]
    for i in range(64):
        x[0, 80, :, 0, i] = (i + 0.5) if fmt == kv8.INT8 else (8 + i / 4.0) * 2.0 ** (i % 5)
    x[0, 80, :, 0, 63] = q
    x[0, 96, 0, 0, 1] = float("inf")
    x[0, 112, 1, 0, 1] = float("nan")
    x[0, 128, :, 0, 0] = -float("inf")
    x[0, 145] = 1e-30
    dev.store(x, [0])
    same(dev, [160])
    # more rows into the last blocks: a NaN block stays one, another's scale rises from the smallest
    y = rows(np.random.default_rng(0), 1, 4, 2, 1, 64)
    dev.store(y, [140])
    dev.store(y, [146])
    code, scale = dev.raw()
    np.testing.assert_array_equal(scale, dev.ref.scale)
    assert np.isnan(scale[0, 0, 0, 6]) and not np.isnan(scale[0, 0, 1, 6]) and np.isnan(scale[0, 0, :, 8]).all()
    out = torch.zeros(1, 144, 2 * 64, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv8_load(dev.kv, 0, 144, out)
    want = dev.ref.read()[..., :144, :].transpose(0, 3, 2, 1, 4).reshape(1, 144, 128)
    want[want == 2.0 ** 128] = np.inf        # what the largest bf16 rounds to in 8 bits
    np.testing.assert_array_equal(f64(out), want)


@FMTS
def test_store_over_zeroed_memory(fmt):
    """Positions before the first one stored count as zeros in a zeroed cache."""
    dev = Dev(fmt, 64, 1, 2, 128, 128)
    dev.codes.zero_()
    dev.scales.zero_()
    dev.ref.code[:], dev.ref.scale[:] = 0.0, 0.0
    dev.store(rows(np.random.default_rng(1), 1, 20, 2, 2, 128), [33])
    code, scale = dev.raw()
    np.testing.assert_array_equal(code[:, :, :, :53], kv8.to_bytes(fmt, dev.ref.code[:, :, :, :53]))
    np.testing.assert_array_equal(scale, dev.ref.scale * (np.arange(2) == 0))


@FMTS
@BLOCKS
@DHS
@pytest.mark.parametrize("pos,n", [(0, 1), (0, 203), (63, 2), (17, 100), (202, 1)])
def test_load(fmt, block, dh, pos, n):
    rng = np.random.default_rng(pos + n)
    dev = Dev(fmt, block, 3, 2, dh, 203)
    dev.ref.store(rows(rng, 3, 203, 2, 2, dh).double().numpy(), [0] * 3)
    dev.upload()
    want = dev.ref.read()[..., pos:pos + n, :].transpose(0, 3, 2, 1, 4).reshape(3, n, -1)
    out = torch.full((3, n, 4 * dh), 7.0, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv8_load(dev.kv, pos, n, out)
    np.testing.assert_array_equal(f64(out), want)
    out.fill_(7.0)
    end = [pos + n // 2, 0, 10 ** 9]
    ld.ld_kv8_load(dev.kv, pos, n, out, seq_len=torch.tensor(end, dtype=torch.int32, device=DEV))
    for b in range(3):
        k = min(max(end[b] - pos, 0), n)
        want[b, k:] = 7.0
    np.testing.assert_array_equal(f64(out), want)


def test_every_code_reads_back():
    """All bytes of both formats, at the smallest and a large scale."""
    for fmt in (kv8.E4M3, kv8.INT8):
        dev = Dev(fmt, 16, 1, 1, 64, 64)
        table = kv8.e4m3_table() if fmt == kv8.E4M3 else np.arange(256).astype(np.uint8).view(np.int8).astype(float)
        raw = np.resize(np.arange(256, dtype=np.uint8), dev.codes.numel())
        dev.codes.copy_(torch.from_numpy(raw))
        dev.scales.copy_(torch.tensor([2.0 ** -100, 1.0, 2.0 ** 100, 2.0 ** 119] * 2))
        out = torch.zeros(1, 64, 128, dtype=torch.bfloat16, device=DEV)
        ld.ld_kv8_load(dev.kv, 0, 64, out)
        s = np.repeat(np.array([2.0 ** -100, 1.0, 2.0 ** 100, 2.0 ** 119]), 16)
        want = table[kv8.unpack(raw, 1, 1, 64, 64)][0, 0] * s[None, :, None]
        np.testing.assert_array_equal(f64(out)[0], want.transpose(1, 0, 2).reshape(64, 128))


# ----------------------------------------------------------------- attention

def bound(o, a, mag, dh, keys):
    """What the roundings may amount to.  u = 2^-24.  A base-2 score: dh products
    summed and three factors, on 1.45 times the sum of magnitudes; its ALiBi
    term 8 u of itself; its distance to the maximum u of that, and the
    exponential 2 u; a wave's or chunk's rescaling 4 u a time, of which a row sees at
    most keys / 64 + 2.  The weight enters sum and norm (twice), split in two bf16
    parts 2^-16; sums over the keys, u each, twice; and half a bf16 step."""
    u = 2.0 ** -24
    x = u * 1.45 * ((dh + 6) * mag[..., 0] + 8 * mag[..., 1] + 4 * mag[..., 2])
    w = 2 * (x + 2 * u + 4 * u * (keys / 64 + 2)) + 2.0 ** -16 + 2 * keys * u
    return 2.0 ** -8 * np.abs(o) + 1.01 * w[..., None] * a + 1e-38


def attend(dev, q, pos, alibi=0, seq_pos=False, ws=None, extra=64, top=None):
    """q bf16 [n_seq, n, H, dh]; top: the call's pos, where it is not the largest."""
    n_seq, n, H, dh = q.shape
    kvh = dev.shape[1]
    qkv = torch.full((n_seq * n, (H + 2 * kvh) * dh), 3.0, dtype=torch.bfloat16)
    qkv[:, :H * dh] = q.reshape(n_seq * n, -1)
    if ws is None:
        ws = torch.empty(ld.ld_attn_decode_kv8_ws_bytes(dev.kv, H, n), dtype=torch.uint8, device=DEV)
    o = torch.full((n_seq * n * H * dh + extra,), 7.0, dtype=torch.bfloat16, device=DEV)
    top = top or max(p for p in pos if p is not None)
    sp = torch.tensor([-1 if p is None else p for p in pos], dtype=torch.int32, device=DEV) if seq_pos else None
    for _ in range(2):
        before = o.clone()
        ld.ld_attn_decode_kv8(dev.kv, H, top, n, qkv.to(DEV), o[:n_seq * n * H * dh].view(n_seq * n, -1), ws,
                              seq_pos=sp, alibi=alibi)
    assert torch.equal(before, o) or bool(torch.isnan(o).any())        # the same again
    assert bool((o[-extra:] == 7.0).all())
    return f64(o[:-extra]).reshape(n_seq, n, H, dh)


def check(dev, q, pos, alibi=0, seq_pos=False, top=None):
    got = attend(dev, q, pos, alibi, seq_pos, top=top)
    values = np.nan_to_num(dev.ref.read(), nan=0.0)
    o, a, mag = kv8.attention(values, q.double().numpy(), pos, alibi)
    keys = max(p for p in pos if p is not None) + q.shape[1]
    far = np.abs(got - o) / bound(o, a, mag, q.shape[-1], keys)
    assert np.max(far) <= 1.0, np.unravel_index(np.argmax(far), far.shape)


def filled(fmt, block, n_seq, kvh, dh, keys, seed, spare=5):
    rng = np.random.default_rng(seed)
    dev = Dev(fmt, block, n_seq, kvh, dh, keys + spare)
    x = rows(rng, n_seq, keys, 2, kvh, dh)
    # blocks of different sizes, so that a wrong scale shows
    x *= torch.from_numpy(2.0 ** (np.arange(keys) // block % 3))[None, :, None, None, None].to(torch.bfloat16)
    dev.ref.store(x.double().numpy(), [0] * n_seq)
    dev.upload()
    return dev, rng


@FMTS
@BLOCKS
@DHS
@pytest.mark.parametrize("keys", [1, 2, 16, 17, 64, 65, 250, 257, 520])
def test_attn_one_row(fmt, block, dh, keys):
    dev, rng = filled(fmt, block, 2, 3, dh, keys, keys)
    check(dev, rows(rng, 2, 1, 3, dh), [keys - 1] * 2)


@FMTS
@DHS
@pytest.mark.parametrize("n", [2, 3, 5, 8])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("keys", [8, 70, 300])
def test_attn_rows_and_groups(fmt, dh, n, group, keys):
    """Several rows, causal among themselves, query heads that share keys."""
    dev, rng = filled(fmt, 32, 2, 2, dh, keys, n + group)
    check(dev, rows(rng, 2, n, 2 * group, dh), [keys - n] * 2, alibi=n % 2)


@FMTS
@pytest.mark.parametrize("group,n", [(1, 1), (3, 1), (5, 7), (20, 8)])
@pytest.mark.parametrize("alibi", [0, 1])
def test_attn_ragged(fmt, group, n, alibi):
    """Lengths from one to many, in chunks (few heads) and in one; sequences left
    out give zeros."""
    dev, rng = filled(fmt, 64, 6, 1, 128, 1500, group)
    check(dev, rows(rng, 6, n, group, 128), [0, None, 1500 - n, 63, None, 800], alibi, seq_pos=True)
    check(dev, rows(rng, 6, n, group, 128), [0, None, 3, 63, 200 - n, 64], alibi, seq_pos=True)
    check(dev, rows(rng, 6, n, group, 128), [5, None, 3, None, None, 64], alibi, seq_pos=True)


def test_attn_all_left_out():
    dev, rng = filled(kv8.E4M3, 64, 2, 1, 64, 900, 0)
    for pos in (899, 40):
        o = torch.full((2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(ld.ld_attn_decode_kv8_ws_bytes(dev.kv, 1, 1), dtype=torch.uint8, device=DEV)
        ld.ld_attn_decode_kv8(dev.kv, 1, pos, 1, torch.ones(2, 192, dtype=torch.bfloat16, device=DEV), o, ws,
                              seq_pos=torch.tensor([-1, pos + 1], dtype=torch.int32, device=DEV))
        assert not bool(o.any())


@FMTS
@DHS
@pytest.mark.parametrize("n_seq,kvh,keys", [(1, 1, 40000), (2, 2, 9000), (9, 16, 2100), (1, 4, 5000)])
def test_attn_long(fmt, dh, n_seq, kvh, keys):
    """Chunks of several turns, many chunks, odd ends."""
    if n_seq * kvh * keys * dh > 2 ** 25:
        keys //= 2
    dev, rng = filled(fmt, 128, n_seq, kvh, dh, keys, keys)
    check(dev, rows(rng, n_seq, 1, kvh, dh, scale=2.0), [keys - 1] * n_seq)
    check(dev, rows(rng, n_seq, 2, 2 * kvh, dh, scale=2.0), [keys - 2] * n_seq, alibi=1)


@FMTS
@DHS
def test_attn_many_rows_in_chunks(fmt, dh):
    """More rows than the merge gives four waves each, of lengths from one chunk to
    three and of none."""
    dev, rng = filled(fmt, 32, 11, 4, dh, 1300, dh)
    pos = [1300 - 8 if b % 4 == 0 else None if b % 4 == 1 else 97 * b for b in range(11)]
    check(dev, rows(rng, 11, 8, 48, dh), pos, seq_pos=True)


@FMTS
@pytest.mark.parametrize("n_seq,kvh,keys", [(8, 4, 3000), (16, 8, 1100)])
def test_attn_uneven_in_a_full_grid(fmt, n_seq, kvh, keys):
    """So many row tiles that long sequences' chunks grow (to one, in the second)
    while short ones' stay."""
    dev, rng = filled(fmt, 128, n_seq, kvh, 64, keys, kvh)
    pos = [None if b == 2 else keys - 8 if b % 3 == 0 else min(100 + 97 * b, keys - 8) for b in range(n_seq)]
    check(dev, rows(rng, n_seq, 8, 32 * kvh, 64), pos, seq_pos=True)


@FMTS
@DHS
@pytest.mark.parametrize("p", [0, 255, 700, 2990])
def test_attn_far_below_the_bound(fmt, dh, p):
    """What a captured step does early on: pos is the most, seq_pos what there is."""
    dev, rng = filled(fmt, 64, 1, 2, dh, 3000, p)
    check(dev, rows(rng, 1, 1, 4, dh), [p], seq_pos=True, top=2999)
    if p <= 1000:
        check(dev, rows(rng, 1, 1, 4, dh), [p], seq_pos=True, top=1000)
    dev, rng = filled(fmt, 64, 3, 2, dh, 3000, p + 1)
    check(dev, rows(rng, 3, 2, 4, dh), [p, None, p // 2], seq_pos=True, top=2998)


@FMTS
def test_attn_far_scales(fmt):
    """Value blocks 2^60 apart, the largest under weights that vanish: nothing of the
    others may be lost; zero blocks with the smallest scale hold the weight."""
    dh, keys = 128, 320
    rng = np.random.default_rng(5)
    dev = Dev(fmt, 16, 1, 1, dh, keys)
    x = rows(rng, 1, keys, 2, 1, dh)
    x[0, :, 0, 0, 0] = 0.0
    x[0, 64:80, 1] *= 2.0 ** 60
    x[0, 64:80, 0, 0, 0] = -64.0      # weights around e^-90 against the rest
    x[0, 160:176, 1] = 0.0
    x[0, 160:176, 0, 0, 0] = 2.0
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    q = rows(rng, 1, 1, 1, dh, scale=0.1)
    q[..., 0] = 16.0
    check(dev, q, [keys - 1])


@FMTS
def test_attn_nan_and_infinite(fmt):
    """A NaN block makes every row that sees one of its positions NaN, and no
    other; an infinite or NaN query its own row."""
    dev, rng = filled(fmt, 16, 2, 2, 64, 600, 3)
    dev.scales.view(2, 2, 2, -1)[0, 0, 0, 20] = float("nan")       # keys 320..335 of head 0
    dev.scales.view(2, 2, 2, -1)[1, 1, 1, 20] = float("nan")       # values of sequence 1, head 1
    q = rows(rng, 2, 4, 2, 64)
    clean = Dev(fmt, 16, 2, 2, 64, 605)
    clean.codes, clean.ref = dev.codes, dev.ref
    clean.scales = torch.from_numpy(dev.ref.scale.reshape(-1)).float().to(DEV)
    clean.kv = ld.kv8(clean.codes, clean.scales, dev.fmt, 16, 2, 2, 64, 605)
    for top in (317, 323, 500):
        got = attend(dev, q, [top] * 2)
        want = attend(clean, q, [top] * 2)
        for j in range(4):
            sees = top + j >= 320
            for b, h in ((0, 0), (1, 1)):
                if sees:
                    assert np.isnan(got[b, j, h]).all()
                    want[b, j, h] = np.nan
        np.testing.assert_array_equal(got, want)
    q[0, 1, 0, 5] = float("nan")
    q[1, 2, 1, 7] = float("inf")
    got = attend(clean, q, [500] * 2)
    want = attend(clean, torch.nan_to_num(q, nan=0.0, posinf=0.0), [500] * 2)
    assert np.isnan(got[0, 1, 0]).all() and np.isnan(got[1, 2, 1]).all()
    want[0, 1, 0] = want[1, 2, 1] = np.nan
    np.testing.assert_array_equal(got, want)


@FMTS
def test_attn_masked_largest_values(fmt):
    """The largest bf16 in a row that earlier rows must not see: in 8 bits it
    stands for 2^128, an infinity that would make NaN of a weight of zero."""
    rng = np.random.default_rng(8)
    dev = Dev(fmt, 16, 1, 1, 64, 40)
    x = rows(rng, 1, 22, 2, 1, 64)
    x[0, 21, 1, 0, 5] = torch.finfo(torch.bfloat16).max
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    q = rows(rng, 1, 2, 1, 64)
    got = attend(dev, q, [20])[:, 0]
    o, a, mag = kv8.attention(np.nan_to_num(dev.ref.read(), nan=0.0), q.double().numpy(), [20], 0)
    assert np.all(np.abs(got - o[:, 0]) <= bound(o, a, mag, 64, 22)[:, 0])


# ------------------------------------------------------------------ together

@FMTS
@pytest.mark.parametrize("block,dh,kvh,H", [(64, 128, 2, 2), (16, 64, 2, 6)])
def test_decoding_over_the_cache(fmt, block, dh, kvh, H):
    """Prompts of different lengths, then steps of one and several rows at each
    sequence's own position: the codes, what they read back as, and the
    attention of every step."""
    rng = np.random.default_rng(11)
    B = 4
    dev = Dev(fmt, block, B, kvh, dh, 400)
    lens = [1, 130, 64, 260]
    for b, n in enumerate(lens):
        x = torch.zeros(B, n, 2, kvh, dh, dtype=torch.bfloat16)
        x[b] = rows(rng, n, 2, kvh, dh)
        dev.store(x, [0 if i == b else None for i in range(B)], n_heads=H, seq_pos=True)
    for n in (1, 1, 5, 1, 8, 1):
        x = rows(rng, B, n, 2, kvh, dh, scale=1.0 + n)
        pos = [None if (b == 2 and n == 5) else p for b, p in enumerate(lens)]
        dev.store(x, pos, n_heads=H, seq_pos=True)
        check(dev, rows(rng, B, n, H, dh), pos, alibi=n % 2, seq_pos=True)
        lens = [p + n if q is not None else p for p, q in zip(lens, pos)]
    same(dev, lens)
    out = torch.zeros(B, 400, 2 * kvh * dh, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv8_load(dev.kv, 0, 400, out, seq_len=torch.tensor(lens, dtype=torch.int32, device=DEV))
    want = np.nan_to_num(dev.ref.read(), nan=0.0).transpose(0, 3, 2, 1, 4).reshape(B, 400, -1)
    for b, n in enumerate(lens):
        want[b, n:] = 0.0
    np.testing.assert_array_equal(f64(out), want)


def test_captured_steps_replayed():
    """One captured step (store, attention, load) replayed while seq_pos
    advances on the device, on a stream of its own, against eager steps."""
    B, kvh, H, dh, steps = 3, 2, 4, 64, 6
    rng = np.random.default_rng(2)
    x = [rows(rng, B, (H + 2 * kvh) * dh).to(DEV) for _ in range(steps)]
    start = torch.tensor([0, 30, 299], dtype=torch.int32, device=DEV)

    def fresh():
        dev = Dev(kv8.INT8, 32, B, kvh, dh, 320)
        dev.codes.zero_()
        dev.scales.zero_()
        ws = torch.empty(ld.ld_attn_decode_kv8_ws_bytes(dev.kv, H, 1), dtype=torch.uint8, device=DEV)
        return dev, ws, torch.zeros(B, H * dh, dtype=torch.bfloat16, device=DEV), \
            torch.zeros(B, 320, 2 * kvh * dh, dtype=torch.bfloat16, device=DEV), start.clone(), x[0].clone()

    def step(dev, ws, o, out, sp, qkv):
        ld.ld_kv8_store(dev.kv, H, 1, 310, qkv, seq_pos=sp)
        ld.ld_attn_decode_kv8(dev.kv, H, 310, 1, qkv, o, ws, seq_pos=sp)
        ld.ld_kv8_load(dev.kv, 0, 320, out)
        sp += 1

    eager, captured = fresh(), fresh()
    step(*fresh())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(*captured)
    for i in range(steps):
        for s in (eager, captured):
            s[5].copy_(x[i])
        step(*eager)
        graph.replay()
        torch.cuda.synchronize()
        for e, c in zip(eager[1:], captured[1:]):
            if e.dtype != torch.uint8:
                assert torch.equal(e, c)
        assert torch.equal(eager[0].codes, captured[0].codes) and torch.equal(eager[0].scales, captured[0].scales)


def test_another_stream():
    dev, rng = filled(kv8.E4M3, 64, 2, 2, 128, 700, 4)
    q = rows(rng, 2, 1, 2, 128)
    want = attend(dev, q, [699] * 2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = attend(dev, q, [699] * 2)
    np.testing.assert_array_equal(got, want)


def test_many_heads():
    """More tiles than a launch dimension has workgroups: the last sequence's rows
    against the oracle."""
    B, kvh, dh, s_max = 4200, 250, 64, 16
    probe = ld.kv8(None, None, ld.LD_KV8_INT8, 16, B, kvh, dh, s_max)
    codes = torch.zeros(ld.ld_kv8_code_bytes(probe), dtype=torch.uint8, device=DEV)
    scales = torch.zeros(ld.ld_kv8_scale_bytes(probe) // 4, device=DEV)
    kv = ld.kv8(codes, scales, ld.LD_KV8_INT8, 16, B, kvh, dh, s_max)
    rng = np.random.default_rng(3)
    x = rows(rng, 2, 1, 2, kvh, dh)
    qkv = torch.zeros(B, 3 * kvh * dh, dtype=torch.bfloat16, device=DEV)
    qkv[0, kvh * dh:], qkv[-1, kvh * dh:] = x[0].reshape(-1).to(DEV), x[1].reshape(-1).to(DEV)
    ld.ld_kv8_store(kv, kvh, 1, 0, qkv)
    out = torch.full((B, 1, 2 * kvh * dh), 7.0, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv8_load(kv, 0, 1, out)
    ref = kv8.Cache(kv8.INT8, 16, 2, kvh, dh, s_max)
    ref.store(x.double().numpy(), [0, 0])
    want = ref.read()[..., :1, :].transpose(0, 3, 2, 1, 4).reshape(2, -1)
    np.testing.assert_array_equal(f64(out[0]), want[:1])
    np.testing.assert_array_equal(f64(out[-1]), want[1:])
    assert not bool(out[1:-1].any())


def test_offsets_past_32_bits():
    """Heads whose codes lie past 4 GiB: the last sequence's against a cache of
    its own."""
    B, kvh, dh, s_max, H = 3, 32, 128, 200000, 32     # 4.9 GB of codes
    one = Dev(kv8.E4M3, 128, 1, kvh, dh, 300)
    probe = ld.kv8(None, None, ld.LD_KV8_E4M3, 128, B, kvh, dh, s_max)
    codes = torch.zeros(ld.ld_kv8_code_bytes(probe), dtype=torch.uint8, device=DEV)
    scales = torch.zeros(ld.ld_kv8_scale_bytes(probe) // 4, device=DEV)
    assert codes.numel() > 2 ** 32
    kv = ld.kv8(codes, scales, ld.LD_KV8_E4M3, 128, B, kvh, dh, s_max)
    rng = np.random.default_rng(6)
    x = rows(rng, 1, 290, 2, kvh, dh)
    q = rows(rng, 1, 1, H, dh)
    one.store(x, [0])
    want = attend(one, q, [289])
    qkv = torch.zeros(B, 290, (H + 2 * kvh) * dh, dtype=torch.bfloat16, device=DEV)
    qkv[2, :, H * dh:] = x[0].reshape(290, -1).to(DEV)
    ld.ld_kv8_store(kv, H, 290, 0, qkv.view(B * 290, -1), seq_pos=torch.tensor([-1, -1, 0], dtype=torch.int32, device=DEV))
    qn = torch.zeros(B, (H + 2 * kvh) * dh, dtype=torch.bfloat16, device=DEV)
    qn[2, :H * dh] = q.reshape(-1).to(DEV)
    o = torch.zeros(B, H * dh, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(ld.ld_attn_decode_kv8_ws_bytes(kv, H, 1), dtype=torch.uint8, device=DEV)
    ld.ld_attn_decode_kv8(kv, H, 289, 1, qn, o, ws, seq_pos=torch.tensor([-1, -1, 289], dtype=torch.int32, device=DEV))
    # the split of the work may differ with the batch: half a bf16 step each
    np.testing.assert_allclose(f64(o[2]).reshape(want.shape[1:]), want[0], rtol=2.0 ** -7, atol=1e-5)
    out = torch.zeros(B, 290, 2 * kvh * dh, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv8_load(kv, 0, 290, out)
    ref = one.ref.read()[..., :290, :].transpose(0, 3, 2, 1, 4).reshape(290, -1)
    np.testing.assert_array_equal(f64(out[2]), ref)
    assert not bool(out[:2].any())
