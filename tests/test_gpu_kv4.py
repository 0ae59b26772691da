"""The 4-bit key/value cache on the HIP path against the float64 oracle: codes and
scales bit for bit, values read back exactly, attention and the positions' weights
within bounds that count their roundings."""
import numpy as np
import pytest
import torch

import paper_2609_05275_amd as ld
from oracle import kv4, kv8
from tests.gpu_util import DEV, f64

pytestmark = pytest.mark.gpu

DHS = pytest.mark.parametrize("dh", [64, 128])
FILL = 0xFF     # a NaN scale: what memory that nobody wrote holds


class Dev:
    """A cache on the GPU whose memory held NaNs, and its oracle."""

    def __init__(self, n_seq, kv_heads, dh, s_max, sums=False):
        self.ref = kv4.Cache(n_seq, kv_heads, dh, s_max)
        self.shape = (n_seq, kv_heads, dh, s_max)
        probe = ld.kv4(None, None, *self.shape)
        self.codes = torch.full((ld.ld_kv4_code_bytes(probe),), FILL, dtype=torch.uint8, device=DEV)
        self.scales = torch.full((ld.ld_kv4_scale_bytes(probe),), FILL, dtype=torch.uint8, device=DEV)
        self.sums = torch.full((n_seq, kv_heads, s_max), 1e9, device=DEV) if sums else None
        self.kv = ld.kv4(self.codes, self.scales, *self.shape, sums=self.sums)

    def scale_view(self, t=None):
        n, kvh, dh, s_max = self.shape
        return (self.scales if t is None else t).view(n, kvh, 2, -1, dh // 32)

    def upload(self, length=None):
        """The oracle's contents of the first length[b] positions to the GPU."""
        n, kvh, dh, s_max = self.shape
        written = kv4.Cache(*self.shape)
        length = length or [s_max] * n
        for b, k in enumerate(length):
            written.code[b, :, :, :k] = 6.0      # a nibble of 7 in every written place
        mask = written.pack()
        packed = self.ref.pack(fill=FILL)
        self.codes.copy_(torch.from_numpy(np.where(mask != 0, packed, FILL).astype(np.uint8)))
        sc = np.full((n, kvh, 2, -(-s_max // 8) * 8, dh // 32), FILL, dtype=np.uint8)
        for b, k in enumerate(length):
            sc[b, :, :, :k] = self.ref.scale[b, :, :, :k]
        self.scales.copy_(torch.from_numpy(sc.reshape(-1)))

    def raw(self):
        n, kvh, dh, s_max = self.shape
        return kv4.unpack(self.codes.cpu().numpy(), n, kvh, dh, s_max), self.scale_view().cpu().numpy()

    def store(self, x, pos, n_heads=None, seq_pos=False, top=None):
        """x [n_seq, n, 2, KV, dh] in bf16; pos: list, None for a sequence left out."""
        n_seq, n, _, kvh, dh = x.shape
        H = n_heads or kvh
        qkv = torch.randn(n_seq, n, (H + 2 * kvh) * dh).to(torch.bfloat16)
        qkv[:, :, H * dh:] = x.reshape(n_seq, n, -1)
        top = top if top is not None else max(p for p in pos if p is not None)
        sp = torch.tensor([-1 if p is None else p for p in pos], dtype=torch.int32, device=DEV) if seq_pos else None
        ld.ld_kv4_store(self.kv, H, n, top, qkv.to(DEV).view(n_seq * n, -1), seq_pos=sp)
        self.ref.store(x.double().numpy(), pos)


def same(dev, spans):
    """Codes and scales of the positions spans[b] = (first, last + 1); the fill elsewhere."""
    code, scale = dev.raw()
    want, ws = np.full(code.shape, 15, np.uint8), np.full(scale.shape, FILL, np.uint8)
    for b, (lo, hi) in enumerate(spans):
        want[b, :, :, lo:hi] = kv4.to_codes(dev.ref.code[b, :, :, lo:hi])
        ws[b, :, :, lo:hi] = dev.ref.scale[b, :, :, lo:hi]
    # (a code of -0 is one of 0; those of a NaN group say nothing)
    zero = lambda c: np.where(c == 8, 0, c)  # noqa: E731
    nan = np.repeat(ws == FILL, 32, -1) & (want != 15)
    np.testing.assert_array_equal(scale, ws)
    np.testing.assert_array_equal(np.where(nan, 0, zero(code)), np.where(nan, 0, zero(want)))


def rows(rng, *shape, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


# ---------------------------------------------------------------- store, load

@DHS
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 16, 64, 129, 200])
@pytest.mark.parametrize("at", [0, 3])
def test_store_prompt(dh, n, at):
    rng = np.random.default_rng(n + at)
    dev = Dev(2, 3, dh, 203)
    x = rows(rng, 2, n, 2, 3, dh)
    x *= torch.from_numpy(2.0 ** rng.integers(-6, 7, (2, n, 2, 3, dh // 32)).repeat(32, -1)).to(torch.bfloat16)
    dev.store(x, [at, at], n_heads=6)
    same(dev, [(at, at + n)] * 2)


@DHS
def test_store_appends_and_overwrites(dh):
    """Rows one call after another, of any number, then others in their places, as
    a verify step does: nothing is left of those."""
    rng = np.random.default_rng(dh)
    dev = Dev(2, 2, dh, 300, sums=True)
    at = 0
    for i, n in enumerate([37, 1, 1, 8, 5, 1, 64, 3, 1, 100, 8]):
        dev.store(rows(rng, 2, n, 2, 2, dh, scale=1.5 ** i), [at, at])
        at += n
        same(dev, [(0, at)] * 2)
    dev.store(rows(rng, 2, 6, 2, 2, dh, scale=1e-3), [at - 58, at - 58])
    same(dev, [(0, at)] * 2)
    assert not bool(dev.sums[:, :, :at].any()) and bool((dev.sums[:, :, at:] == 1e9).all())


@DHS
def test_store_ragged(dh):
    """Each sequence at its own position, some left out; whatever is outside
    [0, pos] counts as left out."""
    rng = np.random.default_rng(5)
    for n in (1, 8, 100):
        dev = Dev(6, 2, dh, 260, sums=True)
        pos = [0, 17, None, 127, 128, None]
        x = rows(rng, 6, n, 2, 2, dh, scale=n)
        sp = torch.tensor([0, 17, -5, 127, 128, 10 ** 9], dtype=torch.int32, device=DEV)
        qkv = torch.cat((torch.zeros(6 * n, 2 * dh, dtype=torch.bfloat16), x.reshape(6 * n, -1)), 1).to(DEV)
        ld.ld_kv4_store(dev.kv, 2, n, 128, qkv, seq_pos=sp)
        dev.ref.store(x.double().numpy(), pos)
        spans = [(0, 0) if p is None else (p, p + n) for p in pos]
        same(dev, spans)
        for b, (lo, hi) in enumerate(spans):
            s = dev.sums[b]
            assert not bool(s[:, lo:hi].any()) and bool((s[:, :lo] == 1e9).all()) and bool((s[:, hi:] == 1e9).all())


def test_store_and_load_extreme_values():
    """Every finite bf16 magnitude, ties, zeros, subnormals, infinities and NaNs."""
    dev = Dev(1, 1, 128, 400)
    bits = torch.arange(0, 0x7F80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)     # 32640: 255 rows of 128
    x = torch.zeros(1, 400, 2, 1, 128, dtype=torch.bfloat16)
    x[0, :255, 0, 0] = bits.view(255, 128)
    x[0, :255, 1, 0] = -bits.view(255, 128)
    # ties of every pair of neighbours, and what lies next to them
    t = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    x[0, 260, :, 0, :21] = torch.cat((t, t * (1 + 2.0 ** -7), t * (1 - 2.0 ** -8))).to(torch.bfloat16)
    x[0, 260, :, 0, 31] = 6.0
    x[0, 261, :, 0, :] = 2.0 ** -130
    x[0, 262, 0, 0, 5] = float("inf")
    x[0, 262, 1, 0, 40] = float("nan")
    x[0, 263, :, 0, 127] = -float("inf")
    x[0, 264, :, 0, 3] = torch.finfo(torch.bfloat16).max
    dev.store(x, [0])
    same(dev, [(0, 400)])
    out = torch.zeros(1, 400, 256, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv4_load(dev.kv, 0, 400, out)
    want = dev.ref.read().transpose(0, 3, 2, 1, 4).reshape(1, 400, 256)
    np.testing.assert_array_equal(f64(out), want)
    assert np.isfinite(want[0, 264]).all() and np.isnan(want[0, 262]).sum() == 64


@DHS
@pytest.mark.parametrize("pos,n", [(0, 1), (0, 203), (63, 2), (17, 100), (202, 1)])
def test_load(dh, pos, n):
    rng = np.random.default_rng(pos + n)
    dev = Dev(3, 2, dh, 203)
    dev.ref.store(rows(rng, 3, 203, 2, 2, dh).double().numpy(), [0] * 3)
    dev.upload()
    want = dev.ref.read()[..., pos:pos + n, :].transpose(0, 3, 2, 1, 4).reshape(3, n, -1)
    out = torch.full((3, n, 4 * dh), 7.0, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv4_load(dev.kv, pos, n, out)
    np.testing.assert_array_equal(f64(out), want)
    out.fill_(7.0)
    end = [pos + n // 2, 0, 10 ** 9]
    ld.ld_kv4_load(dev.kv, pos, n, out, seq_len=torch.tensor(end, dtype=torch.int32, device=DEV))
    for b in range(3):
        want[b, min(max(end[b] - pos, 0), n):] = 7.0
    np.testing.assert_array_equal(f64(out), want)


@DHS
def test_every_code_reads_back(dh):
    dev = Dev(1, 1, dh, 64)
    raw = np.resize(np.random.default_rng(0).permutation(256).astype(np.uint8), dev.codes.numel())
    dev.codes.copy_(torch.from_numpy(raw))
    byte = np.resize(np.array([27, 100, 127, 200, 252, 255], np.uint8), dev.scales.numel())
    dev.scales.copy_(torch.from_numpy(byte))
    out = torch.zeros(1, 64, 2 * dh, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv4_load(dev.kv, 0, 64, out)
    s = kv4.scale_of(byte.reshape(2, 64, dh // 32)).repeat(32, -1)
    want = kv4.from_codes(kv4.unpack(raw, 1, 1, dh, 64))[0, 0] * s
    np.testing.assert_array_equal(f64(out)[0], want.transpose(1, 0, 2).reshape(64, 2 * dh))


# ----------------------------------------------------------------- attention

def weight_bound(mag, dh, keys):
    """What the roundings of a weight may amount to, of itself.  u = 2^-24.  A
    base-2 score: dh products summed and three factors, on 1.45 times the sum of
    magnitudes; its ALiBi term 8 u of itself; its distance to the maximum u of that,
    and the exponential 2 u; a wave's or chunk's rescaling 4 u a time, of which a row
    sees at most keys / 64 + 2.  It enters twice (weight and norm), as the sums over
    the keys do, u each."""
    u = 2.0 ** -24
    x = u * 1.45 * ((dh + 6) * mag[..., 0] + 8 * mag[..., 1] + 4 * mag[..., 2])
    return 2 * (x + 2 * u + 4 * u * (keys / 64 + 2)) + 2 * keys * u


def bound(o, a, mag, dh, keys):
    """And half a bf16 step of the output."""
    return 2.0 ** -8 * np.abs(o) + 1.01 * weight_bound(mag, dh, keys)[..., None] * a + 1e-38


def attend(dev, q, pos, alibi=0, seq_pos=False, ws=None, extra=64, top=None):
    """q bf16 [n_seq, n, H, dh]; top: the call's pos, where it is not the largest.
    The output, and with sums what the call added to them."""
    n_seq, n, H, dh = q.shape
    kvh = dev.shape[1]
    qkv = torch.full((n_seq * n, (H + 2 * kvh) * dh), 3.0, dtype=torch.bfloat16)
    qkv[:, :H * dh] = q.reshape(n_seq * n, -1)
    if ws is None:
        ws = torch.empty(ld.ld_attn_decode_kv4_ws_bytes(dev.kv, H, n), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    o = torch.full((n_seq * n * H * dh + extra,), 7.0, dtype=torch.bfloat16, device=DEV)
    top = top or max(p for p in pos if p is not None)
    sp = torch.tensor([-1 if p is None else p for p in pos], dtype=torch.int32, device=DEV) if seq_pos else None
    sums = []
    for _ in range(2):
        before = o.clone()
        if dev.sums is not None:
            dev.sums.fill_(3.0)
        ld.ld_attn_decode_kv4(dev.kv, H, top, n, qkv.to(DEV), o[:n_seq * n * H * dh].view(n_seq * n, -1), ws,
                              seq_pos=sp, alibi=alibi)
        sums.append(None if dev.sums is None else dev.sums.clone())
    assert torch.equal(before, o) or bool(torch.isnan(o).any())        # the same again
    assert bool((o[-extra:] == 7.0).all())
    if dev.sums is not None:
        assert torch.equal(sums[0].nan_to_num(-1.0), sums[1].nan_to_num(-1.0))
        return f64(o[:-extra]).reshape(n_seq, n, H, dh), f64(sums[0]) - 3.0
    return f64(o[:-extra]).reshape(n_seq, n, H, dh)


def check(dev, q, pos, alibi=0, seq_pos=False, top=None):
    got = attend(dev, q, pos, alibi, seq_pos, top=top)
    values = np.nan_to_num(dev.ref.read(), nan=0.0)
    q64 = q.double().numpy()
    o, a, mag = kv8.attention(values, q64, pos, alibi)
    keys = max(p for p in pos if p is not None) + q.shape[1]
    if dev.sums is not None:
        got, sums = got
        want = kv4.weights(values, q64, pos, alibi)
        # each weight's own error, the rows' sums, and their addition to 3
        R = q.shape[1] * q.shape[2] // dev.shape[1]
        w = np.max(weight_bound(mag, q.shape[-1], keys), initial=0.0) + R * 2.0 ** -24
        far = np.abs(sums - want) / (1.01 * w * want + 2.0 ** -24 * (3.0 + R) + 1e-38)
        assert np.max(far) <= 1.0, np.unravel_index(np.argmax(far), far.shape)
        for b, p in enumerate(pos):      # nothing behind the last position
            assert not sums[b, :, 0 if p is None else p + q.shape[1]:].any()
    far = np.abs(got - o) / bound(o, a, mag, q.shape[-1], keys)
    assert np.max(far) <= 1.0, np.unravel_index(np.argmax(far), far.shape)


def filled(n_seq, kvh, dh, keys, seed, spare=5, sums=False):
    rng = np.random.default_rng(seed)
    dev = Dev(n_seq, kvh, dh, keys + spare, sums=sums)
    x = rows(rng, n_seq, keys, 2, kvh, dh)
    # groups of different sizes, so that a wrong scale shows
    f = 2.0 ** ((np.arange(keys)[:, None] + np.arange(dh // 32)) % 3)
    x *= torch.from_numpy(f.repeat(32, -1))[None, :, None, None].to(torch.bfloat16)
    dev.ref.store(x.double().numpy(), [0] * n_seq)
    dev.upload([keys] * n_seq)
    return dev, rng


@DHS
@pytest.mark.parametrize("sums", [False, True], ids=["plain", "sums"])
@pytest.mark.parametrize("keys", [1, 2, 7, 8, 9, 31, 32, 33, 64, 65, 250, 257, 520])
def test_attn_one_row(dh, keys, sums):
    dev, rng = filled(2, 3, dh, keys, keys, sums=sums)
    check(dev, rows(rng, 2, 1, 3, dh), [keys - 1] * 2)


@DHS
@pytest.mark.parametrize("n", [2, 3, 5, 8])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("keys", [8, 70, 300])
def test_attn_rows_and_groups(dh, n, group, keys):
    """Several rows, causal among themselves, query heads that share keys."""
    dev, rng = filled(2, 2, dh, keys, n + group, sums=True)
    check(dev, rows(rng, 2, n, 2 * group, dh), [keys - n] * 2, alibi=n % 2)


@DHS
@pytest.mark.parametrize("group,n", [(1, 1), (3, 1), (5, 7), (20, 8)])
@pytest.mark.parametrize("alibi", [0, 1])
def test_attn_ragged(dh, group, n, alibi):
    """Lengths from one to many, in chunks (few heads) and in one; sequences left
    out give zeros and draw nothing."""
    dev, rng = filled(6, 1, dh, 1500, group, sums=alibi == 1)
    check(dev, rows(rng, 6, n, group, dh), [0, None, 1500 - n, 63, None, 800], alibi, seq_pos=True)
    check(dev, rows(rng, 6, n, group, dh), [0, None, 3, 63, 200 - n, 64], alibi, seq_pos=True)
    check(dev, rows(rng, 6, n, group, dh), [5, None, 3, None, None, 64], alibi, seq_pos=True)


def test_attn_all_left_out():
    dev, rng = filled(2, 1, 64, 900, 0, sums=True)
    for pos in (899, 40):
        o = torch.full((2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(ld.ld_attn_decode_kv4_ws_bytes(dev.kv, 1, 1), dtype=torch.uint8, device=DEV)
        dev.sums.fill_(2.0)
        ld.ld_attn_decode_kv4(dev.kv, 1, pos, 1, torch.ones(2, 192, dtype=torch.bfloat16, device=DEV), o, ws,
                              seq_pos=torch.tensor([-1, pos + 1], dtype=torch.int32, device=DEV))
        assert not bool(o.any()) and bool((dev.sums == 2.0).all())


@DHS
@pytest.mark.parametrize("n_seq,kvh,keys", [(1, 1, 40000), (2, 2, 9000), (9, 16, 2100), (1, 4, 5000)])
def test_attn_long(dh, n_seq, kvh, keys):
    """Chunks of several turns, many chunks, odd ends."""
    if n_seq * kvh * keys * dh > 2 ** 25:
        keys //= 2
    dev, rng = filled(n_seq, kvh, dh, keys, keys, sums=kvh != 16)
    check(dev, rows(rng, n_seq, 1, kvh, dh, scale=2.0), [keys - 1] * n_seq)
    check(dev, rows(rng, n_seq, 2, 2 * kvh, dh, scale=2.0), [keys - 2] * n_seq, alibi=1)


@DHS
def test_attn_many_rows_in_chunks(dh):
    """Several row tiles, lengths from one chunk to three and none."""
    dev, rng = filled(11, 4, dh, 1300, dh, sums=True)
    pos = [1300 - 8 if b % 4 == 0 else None if b % 4 == 1 else 97 * b for b in range(11)]
    check(dev, rows(rng, 11, 8, 48, dh), pos, seq_pos=True)


@pytest.mark.parametrize("keys,group,n,dh", [(9000, 40, 8, 64), (700, 33, 8, 128), (300, 300, 1, 64), (30000, 1, 1, 128)])
@pytest.mark.parametrize("seq_pos", [False, True], ids=["known", "device"])
def test_attn_sums_of_many_rows_and_chunks(keys, group, n, dh, seq_pos):
    """More rows of a head than their norms are found for at a time, more chunks than lanes
    look at at once."""
    dev, rng = filled(2, 1, dh, keys, group, sums=True)
    check(dev, rows(rng, 2, n, group, dh), [keys - n, None if seq_pos else keys - n], seq_pos=seq_pos)


@pytest.mark.parametrize("n_seq,kvh,keys", [(8, 4, 3000), (16, 8, 1100)])
def test_attn_uneven_in_a_full_grid(n_seq, kvh, keys):
    dev, rng = filled(n_seq, kvh, 64, keys, kvh)
    pos = [None if b == 2 else keys - 8 if b % 3 == 0 else min(100 + 97 * b, keys - 8) for b in range(n_seq)]
    check(dev, rows(rng, n_seq, 8, 32 * kvh, 64), pos, seq_pos=True)


@DHS
@pytest.mark.parametrize("p", [0, 255, 700, 2990])
def test_attn_far_below_the_bound(dh, p):
    """What a captured step does early on: pos is the most, seq_pos what there is."""
    dev, rng = filled(1, 2, dh, 3000, p, sums=True)
    check(dev, rows(rng, 1, 1, 4, dh), [p], seq_pos=True, top=2999)
    dev, rng = filled(3, 2, dh, 3000, p + 1)
    check(dev, rows(rng, 3, 2, 4, dh), [p, None, p // 2], seq_pos=True, top=2998)


def test_attn_far_scales():
    """Value groups 2^60 apart, the largest under weights that vanish: nothing of the
    others may be lost; zero groups with the smallest scale hold the weight."""
    dh, keys = 128, 320
    rng = np.random.default_rng(5)
    dev = Dev(1, 1, dh, keys)
    x = rows(rng, 1, keys, 2, 1, dh)
    x[0, :, 0, 0, :32] = 0.0
    x[0, 64:80, 1] *= 2.0 ** 60
    x[0, 64:80, 0, 0, 0] = -64.0      # weights around e^-90 against the rest
    x[0, 160:176, 1] = 0.0
    x[0, 160:176, 0, 0, 0] = 2.0
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    q = rows(rng, 1, 1, 1, dh, scale=0.1)
    q[..., 0] = 16.0
    check(dev, q, [keys - 1])


def outliers(dh, size, seed):
    """Keys that are zero in two dimensions, where the queries have `size` times what they
    have elsewhere: what the others lose beside it is all there is."""
    rng = np.random.default_rng(seed)
    dev = Dev(1, 1, dh, 300)
    x = rows(rng, 1, 300, 2, 1, dh)
    x[:, :, 0, :, 5] = 0.0
    x[:, :, 0, :, dh - 3] = 0.0
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    q = rng.uniform(0.5, 1.0, (1, 2, 4, dh)) * rng.choice([-1.0, 1.0], (1, 2, 4, dh))
    q[..., 5] *= size
    q[..., dh - 3] *= -size
    return dev, torch.from_numpy(q).to(torch.bfloat16)


@DHS
@pytest.mark.parametrize("size", [1.0, 2.0 ** 6, 2.0 ** 13, 2.0 ** -120, 2.0 ** -13])
def test_attn_query_outliers(dh, size):
    dev, q = outliers(dh, size, 3)
    check(dev, q, [298])


@DHS
@pytest.mark.parametrize("small", [2.0 ** -100, 2.0 ** -112])
def test_attn_small_queries(dh, small):
    """Against keys as large: products around 1."""
    rng = np.random.default_rng(8)
    dev = Dev(1, 2, dh, 120)
    x = rows(rng, 1, 120, 2, 2, dh)
    x[:, :, 0] *= 1.0 / small
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    check(dev, rows(rng, 1, 3, 4, dh) * small, [117])


@DHS
@pytest.mark.parametrize("size", [2.0 ** 15, 2.0 ** 16])
def test_attn_query_outliers_beyond(dh, size):
    """Below 2^-14 of its 32 dimensions' largest, a query's may be off by 2^-22 of that: a
    base-2 score by 1.45 / sqrt(dh) times the sum of |k| times it, which enters twice, in a
    weight and in the norm (4^x - 1 < 2 x for the x < 1/2 here)."""
    dev, q = outliers(dh, size, 4)
    got = attend(dev, q, [298])
    values, q64 = dev.ref.read(), q.double().numpy()
    o, a, mag = kv8.attention(values, q64, [298], 0)
    top = np.abs(q64).reshape(*q64.shape[:-1], dh // 32, 32).max(-1).repeat(32, -1)      # [1, n, H, dh]
    off = 1.45 / np.sqrt(dh) * 2.0 ** -22 * (top @ np.abs(values[0, 0, 0]).T).max(-1)
    assert off.max() < 0.5
    w = 2 * off[..., None] * a
    assert np.max(np.abs(got - o) / (bound(o, a, mag, dh, 300) + 1.01 * (1 + 2.0 ** -8) * w)) <= 1.0


@DHS
def test_attn_values_that_cancel(dh):
    """Equal weights on values that sum to almost nothing: what a weight rounded to
    fewer bits would leave shows."""
    keys = 256
    dev = Dev(1, 1, dh, keys)
    x = torch.zeros(1, keys, 2, 1, dh, dtype=torch.bfloat16)
    x[0, :, 0, 0, 0] = torch.from_numpy(np.random.default_rng(0).standard_normal(keys)).to(torch.bfloat16)
    x[0, 0::2, 1], x[0, 1::2, 1] = 6.0, -6.0
    x[0, 1::2, 0, 0, 0] = x[0, 0::2, 0, 0, 0]
    x[0, keys - 1, 1, 0] = -4.0
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    q = torch.zeros(1, 1, 1, dh, dtype=torch.bfloat16)
    q[..., 0] = 3.0
    got = attend(dev, q, [keys - 1])
    o, a, mag = kv8.attention(dev.ref.read(), q.double().numpy(), [keys - 1], 0)
    # one step of float32 for each key summed, both sums, and half a bf16 step
    assert np.all(np.abs(got - o) <= 2.0 ** -8 * np.abs(o) + 2 * keys * 2.0 ** -24 * a)


@DHS
def test_attn_nan(dh):
    """A NaN group of keys makes every row that sees its position NaN, one of values
    its 32 dimensions, and nothing else, in places that later rows see and earlier
    ones do not too; a NaN query its own row."""
    dev, rng = filled(2, 2, dh, 600, 3, sums=True)
    clean = Dev(2, 2, dh, 605, sums=True)
    clean.codes.copy_(dev.codes)
    clean.scales.copy_(dev.scales)
    dev.scale_view()[0, 0, 0, 323, 1] = FILL
    dev.scale_view()[1, 1, 1, 323, 1] = FILL
    q = rows(rng, 2, 4, 2, dh)
    for top in (317, 319, 320, 321, 322, 323, 500):
        got, gs = attend(dev, q, [top] * 2)
        want, ws = attend(clean, q, [top] * 2)
        for j in range(4):
            if top + j >= 323:
                want[0, j, 0] = np.nan
                want[1, j, 1, 32:64] = np.nan
        np.testing.assert_array_equal(got, want)
        # sums: NaN where a NaN row sees, as they were elsewhere
        seen = top + 4 if top + 3 >= 323 else 0
        assert np.isnan(gs[0, 0, :seen]).all() or seen == 0
        np.testing.assert_array_equal(gs[1], ws[1])
        np.testing.assert_array_equal(gs[0, 1], ws[0, 1])
        np.testing.assert_array_equal(gs[0, 0, seen:], ws[0, 0, seen:])
    q[0, 1, 0, 5] = float("nan")
    got, _ = attend(clean, q, [500] * 2)
    want, _ = attend(clean, torch.nan_to_num(q, nan=0.0), [500] * 2)
    assert np.isnan(got[0, 1, 0]).all()
    want[0, 1, 0] = np.nan
    np.testing.assert_array_equal(got, want)


def test_attn_largest_values():
    """The largest bf16s are held as a finite 6 2^125, and hurt no row that does not see
    them."""
    rng = np.random.default_rng(8)
    dev = Dev(1, 1, 64, 40)
    x = rows(rng, 1, 22, 2, 1, 64)
    x[0, 21, 1, 0, 5] = torch.finfo(torch.bfloat16).max
    dev.ref.store(x.double().numpy(), [0])
    dev.upload([22])
    q = rows(rng, 1, 2, 1, 64)
    check(dev, q, [20])


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dh,kvh,H", [(128, 2, 2), (64, 2, 6)])
def test_decoding_over_the_cache(dh, kvh, H):
    """Prompts of different lengths, then steps of one and several rows at each
    sequence's own position: the codes, what they read back as, the attention of
    every step, and the sums that the steps leave."""
    rng = np.random.default_rng(11)
    B = 4
    dev = Dev(B, kvh, dh, 400, sums=True)
    lens = [1, 130, 64, 260]
    for b, n in enumerate(lens):
        x = torch.zeros(B, n, 2, kvh, dh, dtype=torch.bfloat16)
        x[b] = rows(rng, n, 2, kvh, dh)
        dev.store(x, [0 if i == b else None for i in range(B)], n_heads=H, seq_pos=True)
    total = np.zeros((B, kvh, 400))
    ws = torch.empty(ld.ld_attn_decode_kv4_ws_bytes(dev.kv, H, 8), dtype=torch.uint8, device=DEV)
    for n in (1, 1, 5, 1, 8, 1):
        x = rows(rng, B, n, 2, kvh, dh, scale=1.0 + n)
        pos = [None if (b == 2 and n == 5) else p for b, p in enumerate(lens)]
        dev.store(x, pos, n_heads=H, seq_pos=True)
        keep = dev.sums.clone()
        q = rows(rng, B, n, H, dh)
        check(dev, q, pos, alibi=n % 2, seq_pos=True)
        dev.sums.copy_(keep)
        sp = torch.tensor([-1 if p is None else p for p in pos], dtype=torch.int32, device=DEV)
        qkv = torch.zeros(B * n, (H + 2 * kvh) * dh, dtype=torch.bfloat16)
        qkv[:, :H * dh] = q.view(B * n, -1)
        ld.ld_attn_decode_kv4(dev.kv, H, max(p for p in pos if p is not None), n, qkv.to(DEV),
                              torch.zeros(B * n, H * dh, dtype=torch.bfloat16, device=DEV), ws, seq_pos=sp, alibi=n % 2)
        total += kv4.weights(np.nan_to_num(dev.ref.read()), q.double().numpy(), pos, n % 2)
        lens = [p + n if q is not None else p for p, q in zip(lens, pos)]
    same(dev, [(0, n) for n in lens])
    got = f64(dev.sums)
    for b, n in enumerate(lens):
        np.testing.assert_allclose(got[b, :, :n], total[b, :, :n], rtol=2e-4, atol=1e-6)
        assert np.all(got[b, :, n:] == 1e9)


def test_captured_steps_replayed():
    """One captured step (store, attention with sums, load) replayed while seq_pos
    advances on the device, against eager steps."""
    B, kvh, H, dh, steps = 3, 2, 4, 64, 6
    rng = np.random.default_rng(2)
    x = [rows(rng, B, (H + 2 * kvh) * dh).to(DEV) for _ in range(steps)]
    start = torch.tensor([0, 30, 299], dtype=torch.int32, device=DEV)

    def fresh():
        dev = Dev(B, kvh, dh, 320, sums=True)
        dev.codes.zero_()
        dev.scales.fill_(127)
        dev.sums.zero_()
        ws = torch.empty(ld.ld_attn_decode_kv4_ws_bytes(dev.kv, H, 1), dtype=torch.uint8, device=DEV)
        return dev, ws, torch.zeros(B, H * dh, dtype=torch.bfloat16, device=DEV), \
            torch.zeros(B, 320, 2 * kvh * dh, dtype=torch.bfloat16, device=DEV), start.clone(), x[0].clone()

    def step(dev, ws, o, out, sp, qkv):
        ld.ld_kv4_store(dev.kv, H, 1, 310, qkv, seq_pos=sp)
        ld.ld_attn_decode_kv4(dev.kv, H, 310, 1, qkv, o, ws, seq_pos=sp)
        ld.ld_kv4_load(dev.kv, 0, 320, out)
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
        for e, c in zip(eager[2:], captured[2:]):
            assert torch.equal(e, c)
        assert torch.equal(eager[0].codes, captured[0].codes) and torch.equal(eager[0].scales, captured[0].scales)
        assert torch.equal(eager[0].sums, captured[0].sums)


def test_another_stream():
    dev, rng = filled(2, 2, 128, 700, 4, sums=True)
    q = rows(rng, 2, 1, 2, 128)
    want, ws = attend(dev, q, [699] * 2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got, gs = attend(dev, q, [699] * 2)
    np.testing.assert_array_equal(got, want)
    np.testing.assert_array_equal(gs, ws)


@pytest.mark.parametrize("n_seq,kvh,s_max", [(70, 8, 65536), (1, 4, 5000000)])
def test_past_32_bits(n_seq, kvh, s_max):
    """Caches whose last rows lie behind 2^32 bytes (or their scales behind 2^31)."""
    dh = 128
    probe = ld.kv4(None, None, n_seq, kvh, dh, s_max)
    if n_seq > 1:
        assert ld.ld_kv4_code_bytes(probe) > 2 ** 32
    dev = Dev.__new__(Dev)
    dev.shape = (n_seq, kvh, dh, s_max)
    dev.codes = torch.zeros(ld.ld_kv4_code_bytes(probe), dtype=torch.uint8, device=DEV)
    dev.scales = torch.full((ld.ld_kv4_scale_bytes(probe),), 127, dtype=torch.uint8, device=DEV)
    kv = ld.kv4(dev.codes, dev.scales, n_seq, kvh, dh, s_max)
    rng = np.random.default_rng(0)
    n, pos = 3, s_max - 3
    qkv = rows(rng, n_seq * n, 3 * kvh * dh).to(DEV)
    ld.ld_kv4_store(kv, kvh, n, pos, qkv)
    out = torch.zeros(n_seq, n, 2 * kvh * dh, dtype=torch.bfloat16, device=DEV)
    ld.ld_kv4_load(kv, pos, n, out)
    last = qkv.view(n_seq, n, 3 * kvh * dh)[-1, :, kvh * dh:].double().cpu().numpy()
    code, byte = kv4.quantise(last)
    np.testing.assert_array_equal(f64(out[-1]), code * np.repeat(kv4.scale_of(byte), 32, -1))
    # all other keys and values are zeros: weights of e^0 against these rows'
    o = torch.zeros(n_seq * n, kvh * dh, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(ld.ld_attn_decode_kv4_ws_bytes(kv, kvh, n), dtype=torch.uint8, device=DEV)
    ld.ld_attn_decode_kv4(kv, kvh, pos, n, qkv * 4, o, ws)
    x = f64(out[-1]).reshape(n, 2, kvh, dh)
    q = (4 * qkv.view(n_seq, n, 3, kvh, dh)[-1, :, 0].double()).cpu().numpy()
    got = f64(o).reshape(n_seq, n, kvh, dh)[-1]
    for j in range(n):
        for h in range(kvh):
            s = x[:j + 1, 0, h] @ q[j, h] / np.sqrt(dh)
            m = max(s.max(), 0.0)
            w = np.exp(s - m)
            want = w @ x[:j + 1, 1, h] / (w.sum() + pos * np.exp(-m))
            a = w @ np.abs(x[:j + 1, 1, h]) / (w.sum() + pos * np.exp(-m))
            # the norm sums pos equal terms in waves and chunks of them: at most 2^13 in a row
            assert np.all(np.abs(got[j, h] - want) <= 2.0 ** -8 * np.abs(want) + a * (2 * 2.0 ** 13 * 2.0 ** -24 + 1e-4) + 1e-38)


def test_two_captured_calls_share_a_workspace():
    """Attention with sums over two caches, in graphs over one workspace."""
    devs = [filled(*sh, sums=True)[0] for sh in ((2, 2, 64, 700, 1), (1, 2, 128, 2500, 2))]
    calls, graphs = [], []
    ws = torch.empty(max(ld.ld_attn_decode_kv4_ws_bytes(d.kv, 8, 3) for d in devs), dtype=torch.uint8, device=DEV)
    rng = np.random.default_rng(6)
    for d, keys in zip(devs, (700, 2500)):
        n_seq, kvh, dh = d.kv.n_seq, d.kv.n_kv_heads, d.kv.d_head
        qkv = rows(rng, n_seq * 3, (8 + 2 * kvh) * dh).to(DEV)
        o = torch.zeros(n_seq * 3, 8 * dh, dtype=torch.bfloat16, device=DEV)
        call = lambda d=d, qkv=qkv, o=o, keys=keys: ld.ld_attn_decode_kv4(d.kv, 8, keys - 3, 3, qkv, o, ws)  # noqa: E731
        call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
        calls.append((d, qkv, o, call))
    for i in range(3):
        for d, qkv, _, _ in calls:
            qkv.copy_(rows(rng, *qkv.shape))
            d.sums.zero_()
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        got = [(o.clone(), d.sums.clone()) for d, _, o, _ in calls]
        for (d, _, o, call), (want_o, want_s) in zip(calls, got):
            d.sums.zero_()
            call()
            assert torch.equal(o, want_o) and torch.equal(d.sums, want_s)
