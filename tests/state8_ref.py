"""Adam's 8-bit states on the host: the format and the step from their definitions, in numpy (fp32 where the state's
arithmetic is defined in fp32, fp64 otherwise)."""
import numpy as np

SEG = 1024
M32 = 0xFFFFFFFF
F = np.float32


def mix(x):
    x = np.asarray(x, dtype=np.uint64)
    for shift, odd in ((16, 0x9E3779B1), (15, 0x6A09E667), (13, 0x5BE0CD19)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(odd)) & np.uint64(M32)
    return x ^ (x >> np.uint64(16))


def key(seed, step):
    x = (seed * 0x9E3779B1 + step * 0x85A308D3) & M32
    x = ((x ^ (x >> 16)) * 0x6A09E667) & M32
    return x ^ (x >> 15)


def _number(e, f, bias):
    """(1 + f/8) 2^(e - bias), or f/8 2^(1 - bias) where e is 0."""
    return np.where(e == 0, np.ldexp(f / 8.0, 1 - bias), np.ldexp(1 + f / 8.0, e.astype(np.int64) - bias))


M_VALUES = _number(np.arange(128) // 8, np.arange(128) % 8, 7)          # of the codes without a sign
V_VALUES = _number(np.arange(256) // 8, np.arange(256) % 8, 31)


def units(scale):
    scale = np.asarray(scale, dtype=np.int64)
    return np.where(scale == 255, np.nan, np.where(scale == 0, 0.0, np.ldexp(1.0, scale - 127)))


def decode(q8, s8, idx):
    """m, v in fp64 (exact)."""
    code, scale = q8.reshape(-1, 2), s8.reshape(-1, 2)[idx // SEG]
    m = M_VALUES[code[:, 0] & 127] * np.where(code[:, 0] >= 128, -1.0, 1.0) * units(scale[:, 0])
    return m, V_VALUES[code[:, 1]] * units(scale[:, 1])


def _exponent_field(x):
    return (np.abs(x).astype(F).view(np.uint32) >> 23).astype(np.int64)


def _up_or_down(values, a, noise):
    """The code of the value below a, or of the one above where a's place between the two plus the noise reaches 1."""
    low = np.clip(np.searchsorted(values, a, side="right") - 1, 0, len(values) - 1)
    gap = np.where(low + 1 < len(values), values[np.minimum(low + 1, len(values) - 1)] - values[low], 1.0)
    # the place is what is left of a's 23 bits of mantissa behind the code's three: 20 bits
    place = np.floor((a - values[low]) / gap * 2.0 ** 20) / 2.0 ** 20
    return low + (place + noise >= 1.0)


def encode(m, v, idx, segments, noise_m, noise_v):
    """q8, s8 of fp32 m and v; the noise is a fraction below 1."""
    seg = idx // SEG
    top_m, top_v = np.zeros(segments, np.int64), np.zeros(segments, np.int64)
    np.maximum.at(top_m, seg, _exponent_field(m))
    np.maximum.at(top_v, seg, _exponent_field(v))
    sm = np.where(top_m == 255, 255, np.maximum(top_m - 7, 1))
    sv = np.where(top_v >= 253, 255, top_v + 1)
    with np.errstate(invalid="ignore", over="ignore"):
        am = np.where(sm[seg] == 255, 0.0, np.abs(m.astype(np.float64)) * np.ldexp(1.0, 127 - sm[seg]))
        av = np.where(sv[seg] == 255, 0.0, v.astype(np.float64) * np.ldexp(1.0, 127 - sv[seg]))
    cm = _up_or_down(M_VALUES, am, noise_m) | np.where(np.signbit(m), 128, 0)
    cv = _up_or_down(V_VALUES, av, noise_v)
    cv = np.where((v > 0) & (cv == 0), 1, cv)
    cm, cv = np.where(sm[seg] == 255, 0, cm), np.where(sv[seg] == 255, 0, cv)
    pair = lambda a, b: np.stack([a, b], 1).astype(np.uint8).reshape(-1)
    return pair(cm, cv), pair(sm, sv)


def noises(idx, rng_offset, seed, step):
    h = mix(((idx.astype(np.int64) + rng_offset) & M32) ^ key(seed, step))
    return ((h & np.uint64(0xFFFF)).astype(np.float64) * 16 + 8) / 2 ** 20, ((h >> np.uint64(16)).astype(np.float64) * 16 + 8) / 2 ** 20


def step(g16, idx, p, q8, s8, inv_scale, cfg, seed, rng_offset=0, coef=1.0):
    """One step in place on p (fp32), q8, s8 from the compressed fp16 gradient; p's update in fp64, rounded once."""
    b1, b2 = F(cfg["beta1"]), F(cfg["beta2"])
    omb1, omb2 = F(1.0 - float(b1)), F(1.0 - float(b2))
    m, v = decode(q8, s8, idx)
    m, v = m.astype(F), v.astype(F)
    with np.errstate(invalid="ignore", over="ignore"):
        g = g16.astype(F) * F(inv_scale) * F(coef)
        wd = cfg.get("weight_decay", 0.0)
        if wd and not cfg.get("decoupled_wd", 0):
            g = (np.float64(F(wd)) * p.astype(np.float64) + g).astype(F)
        m = m * b1 + g * omb1
        v = v * b2 + (g * omb2) * g
        t = cfg["step"]
        m64, v64, p64 = m.astype(np.float64), v.astype(np.float64), p.astype(np.float64)
        upd = m64 / (1 - float(b1) ** t) / (np.sqrt(v64 / (1 - float(b2) ** t)) + float(F(cfg["eps"])))
        if wd and cfg.get("decoupled_wd", 0):
            upd = upd + float(F(wd)) * p64
        p[:] = (p64 - float(F(cfg["lr"])) * upd).astype(F)
    nm, nv = noises(idx, rng_offset, seed, t)
    q, s = encode(m, v, idx, s8.size // 2, nm, nv)
    q8[:], s8[:] = q, s
    return m, v
