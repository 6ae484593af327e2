"""Plain definitions of the network operators in 64 bits (torch on the CPU, numpy), for the tests."""
import numpy as np
import torch

EPS32 = 2.0 ** -24  # half a unit in the last place of float32
EPS16 = 2.0 ** -8   # of bfloat16 (8 significant bits)


def rms_norm(h, w, eps):
    return h / (h.square().mean(1, keepdim=True) + eps).sqrt() * w


def scale_bytes(top):
    """The block scale's byte: the least power of two s >= 2^-127 with top <= 448 s."""
    top = np.asarray(top, dtype=np.float64)
    e = np.full(top.shape, -127.0)
    pos = top > 0
    e[pos] = np.ceil(np.log2(top[pos] / 448.0))
    e[pos] += top[pos] > 448.0 * 2.0 ** e[pos]          # (log2 rounds)
    e[pos] -= top[pos] <= 448.0 * 2.0 ** (e[pos] - 1)
    return (np.clip(e, -127, None) + 127).astype(np.uint8)


def quantize(x, tile):
    """float64 [rows, cols] -> codes' values float64 (NaN for what is not finite), scale bytes."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    fin = np.where(np.isfinite(x), np.abs(x), 0.0)
    sr, sc = -(-rows // tile), -(-cols // 128)
    bytes_ = np.zeros((sr, sc), np.uint8)
    for i in range(sr):
        for j in range(sc):
            bytes_[i, j] = scale_bytes(fin[i * tile:(i + 1) * tile, j * 128:(j + 1) * 128].max())
    s = 2.0 ** (np.repeat(np.repeat(bytes_.astype(np.float64), tile, 0)[:rows], 128, 1)[:, :cols] - 127.0)
    t = x / s
    with np.errstate(divide="ignore", invalid="ignore"):
        ulp = 2.0 ** (np.maximum(np.floor(np.log2(np.where(t == 0, 1.0, np.abs(t)))), -6.0) - 3.0)
        v = np.rint(t / ulp) * ulp  # rint: ties to even, as e4m3's last bit
    return np.where(np.isfinite(x), v, np.nan), bytes_


def values(b):
    """What a Blocks8 stands for, float64 on the CPU."""
    v, s = b.values.cpu().double(), b.scales.cpu().contiguous().view(torch.uint8).double()
    s = torch.exp2(s - 127).repeat_interleave(b.tile, 0)[:v.shape[0]].repeat_interleave(128, 1)[:, :v.shape[1]]
    return v * s


GOLDEN, MASK = 0x9E3779B97F4A7C15, (1 << 64) - 1


def mix64(z):
    z = np.asarray(z, dtype=np.uint64)
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def key_fold(h, v):
    return int(mix64(np.uint64((h + (v + 1) * GOLDEN) & MASK)))


def random16(key, n):
    """Two 16-bit random numbers for each of n values."""
    pairs = np.arange(1, (n + 1) // 2 + 1, dtype=np.uint64)
    with np.errstate(over="ignore"):
        z = mix64(np.uint64(key) + pairs * np.uint64(GOLDEN))
    z = np.stack([z & np.uint64(0xFFFFFFFF), z >> np.uint64(32)], 1).reshape(-1)[:n].astype(np.uint32)
    return z & 0xFFFF, z >> 16


def e4m3_values():
    """The 127 magnitudes by code."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


def round_random(t, r16, least):
    """float32 |t| <= 448 -> code: up with probability (distance from the lower value) / (their distance), to 16 bits."""
    val = e4m3_values()
    a = np.abs(t.astype(np.float64))
    lower = np.clip(np.searchsorted(val, a, side="right") - 1, 0, 126)
    gap = np.where(lower < 126, val[np.minimum(lower + 1, 126)] - val[lower], 1.0)
    share = (a - val[lower]) / gap  # of 2^20 in the code's remaining bits
    rest = np.floor(share * 2.0 ** 20 + 1e-9).astype(np.int64)
    code = lower + ((rest + (r16.astype(np.int64) << 4)) >> 20)
    code = np.where((a > 0) & (code < least), least, code)
    return (code | np.where(t < 0, 128, 0)).astype(np.uint8)


def decode(code):
    v = e4m3_values()[np.minimum(code & 127, 126)]
    return np.where(code & 128, -v, v).astype(np.float32)


def blocks(x):
    """Padded to [blocks, 128] with zeros."""
    n = len(x)
    return np.concatenate([x, np.zeros(-n % 128, x.dtype)]).reshape(-1, 128)


def adam8(g, m, ms, v, vs, beta1, beta2, key):
    """The moments' update in float32, each operation rounded: (m, v, m codes, m scales, v codes, v scales)."""
    f = np.float32
    n = len(g)
    b1, b2, c1, c2 = f(beta1), f(beta2), f(1 - beta1), f(1 - beta2)
    g, cm, cv = blocks(g.astype(f)), blocks(decode(m)), blocks(decode(v))
    mn = cm * ms[:, None] * b1 + g * c1
    old = np.maximum(vs * b2, f(2.0 ** -100))
    vn = cv * old[:, None] + g * g * c2
    mtop, vtop = np.abs(mn).max(1), vn.max(1)
    ms2 = np.maximum(2.0 ** (scale_bytes(mtop).astype(np.float64) - 127), 2.0 ** -100).astype(f)
    # the decayed scale times the power of two that brings the largest into (224, 448]
    vs2 = old.copy()
    for i in range(len(old)):
        s = float(old[i]) / 2.0 ** np.floor(np.log2(float(old[i])))  # mantissa in [1, 2)
        e = -100
        if vtop[i] > 0:
            e = int(np.floor(np.log2(float(vtop[i])))) - 12
            while float(vtop[i]) > 448.0 * s * 2.0 ** e:
                e += 1
        vs2[i] = f(s * 2.0 ** max(e, -100))
    rm, rv = random16(key, mn.size)
    code_m = round_random((mn * (f(1) / ms2)[:, None]).reshape(-1), rm, 0)
    code_v = round_random((vn * (f(1) / vs2)[:, None]).reshape(-1), rv, 1)
    return mn.reshape(-1)[:n], vn.reshape(-1)[:n], code_m[:n], ms2, code_v[:n], vs2
