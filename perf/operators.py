"""The expert-stage operators, case by case: routing slots to experts, moving rows there and back
(with the gradients), products with 4-bit group-scaled weights, and quantisation to that format.

``run`` computes a case in plain torch operations in 32 bits where ``own`` is false, and through the
library's calls where it is true; ``exact`` computes the same from the definition in 64 bits.

The 4-bit format (the library's storage, so that neither side lays weights out again): tiles of 128
output rows x 128 inputs, ``q`` uint8 [E][N/128][K/128][128][64], ``scale`` bfloat16 [E][groups][Npad],
``zero`` uint8 [E][groups][Npad] or None (then 8); a weight is (q - zero) * scale.  In the 64 bytes of row
r of a tile, the 16-byte piece at position p belongs to quarter t = p ^ ((r >> 1) & 3); its 4-byte word b
holds inputs 32 b + 8 t + (0..7), as four bytes (k0 | k2 << 4), (k4 | k6 << 4), (k1 | k3 << 4),
(k5 | k7 << 4).  Rows and inputs past N and K are padding with scale 0.
"""
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _lib():
    import paper_2512_19342_b200 as bls
    return bls


# ---------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one request of one token in a decoding loop: latency alone
        dict(name="route one token", op="route", n=1, k=8, E=64, left_out=0.0),
        # a prefill batch over many experts, some tokens masked out
        dict(name="route a long batch", op="route", n=50001, k=8, E=256, left_out=0.03),
        # a small decoding batch: rows to the experts and the weighted sum back
        dict(name="move 16 tokens", op="move", n=16, k=4, D=1024, dtype="bf16", left_out=0.0, train=False),
        # one training step's movements of a micro-batch whose width no 16-byte piece divides; a tenth of the slots dropped
        dict(name="move odd fp32 step", op="move", n=3001, k=3, D=1531, dtype="f32", left_out=0.1, train=True),
        # the largest training step: forward and backward of dispatch and combine
        dict(name="move a large step", op="move", n=16384, k=8, D=2048, dtype="bf16", left_out=0.02, train=True),
        # the matrix-vector product of a decoding step
        dict(name="w4 one row", op="linear", rows=1, N=4096, K=4096, group=128, zero=False, dtype="bf16", act=0, bias=False),
        # a handful of requests, ragged sizes, small groups with zero points
        dict(name="w4 13 rows ragged", op="linear", rows=13, N=5003, K=2407, group=32, zero=True, dtype="f16", act=1, bias=True),
        # a long prompt through a large layer: compute-bound
        dict(name="w4 long prompt", op="linear", rows=8192, N=8192, K=4096, group=128, zero=False, dtype="bf16", act=0, bias=True),
        # one token's experts: 8 of 64 matrices are read
        dict(name="experts one token", op="experts", rows=8, E=64, active=8, N=2048, K=1024, group=64, zero=False, dtype="bf16", act=1, bias=True),
        # a training-free prefill over all experts, uneven loads
        dict(name="experts long batch", op="experts", rows=16000, E=32, active=32, N=2048, K=2048, group=64, zero=True, dtype="bf16", act=1, bias=True),
        # one small ragged layer turned into 4 bits and looked at again
        dict(name="quantize a layer", op="quantize", E=1, N=1000, K=1023, group=32, zero=True, dtype="f32"),
        # the experts of one stage at load time
        dict(name="quantize experts", op="quantize", E=16, N=4096, K=2048, group=128, zero=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "move", "move", "linear", "linear", "linear", "experts", "experts", "quantize"])
    if op == "route":
        return dict(op=op, n=_log(rng, 1, 50000), k=rng.randint(1, 8), E=_log(rng, 8, 256), left_out=rng.choice([0.0, 0.03, 0.5]))
    if op == "move":
        k = rng.randint(1, 8)
        D = _log(rng, 64, 4096) if rng.random() < 0.5 else 8 * _log(rng, 8, 512)
        n = min(_log(rng, 1, 16384), 16384 * 8 * 2048 // (2 * k * D))
        return dict(op=op, n=n, k=k, D=D, dtype=rng.choice(["bf16", "f16", "f32"]), left_out=rng.choice([0.0, 0.1]),
                    train=rng.random() < 0.6)
    group, zero, dtype = rng.choice([32, 64, 128]), rng.random() < 0.5, rng.choice(["bf16", "f16"])
    if op == "quantize":
        E = _log(rng, 1, 16)
        N = _log(rng, 64, 4096)
        K = min(_log(rng, 64, 8192), 16 * 4096 * 2048 // (E * N))
        return dict(op=op, E=E, N=N, K=K, group=group, zero=zero, dtype=rng.choice(["bf16", "f16", "f32"]))
    more = dict(group=group, zero=zero, dtype=dtype, act=rng.choice([0, 1, 2]), bias=rng.random() < 0.5)
    step = rng.choice([1, 8, 64])                    # odd widths, whole 16-byte pieces, whole tiles
    if op == "linear":
        N, K = (step * max(1, _log(rng, 256, 8192) // step) for _ in range(2))
        rows = min(_log(rng, 1, 8192), 8192 * 8192 * 4096 // (N * K))
        return dict(op=op, rows=rows, N=N, K=K, **more)
    E = _log(rng, 2, 64)
    N, K = (step * max(1, _log(rng, 256, 2048) // step) for _ in range(2))
    rows = _log(rng, 1, 16000)
    return dict(op=op, rows=rows, E=E, active=min(rows, rng.randint(max(1, E // 4), E)), N=N, K=K, **more)


# ---------------------------------------------------------------------------------------- inputs

def _experts(gen, n, k, E, left_out):
    """k different experts for each token, popular ones more often; -1 where a slot or a whole token is left out."""
    logits = torch.rand(n, E, device="cuda", generator=gen).log_().neg_().log_().neg_()      # Gumbel noise
    logits += 0.7 * torch.randn(E, device="cuda", generator=gen)
    e = logits.topk(min(k, E), dim=1).indices.to(torch.int32)
    if left_out:
        e = torch.where(torch.rand(e.shape, device="cuda", generator=gen) < left_out / 2, -1, e)
        e = torch.where(torch.rand(n, 1, device="cuda", generator=gen) < left_out / 2, -1, e).to(torch.int32)
    return e.contiguous()


def _plain_route(expert, E):
    flat = expert.reshape(-1).long()
    here = (flat >= 0) & (flat < E)
    key = torch.where(here, flat, E)
    sort = torch.sort(key, stable=True)
    total = here.sum()
    at = torch.arange(flat.numel(), device=flat.device)
    order = torch.where(at < total, sort.indices, -1).to(torch.int32)
    place = torch.empty_like(at)
    place[sort.indices] = at
    place = torch.where(here, place, -1).to(torch.int32).reshape(expert.shape)
    offsets = torch.searchsorted(sort.values, torch.arange(E + 1, device=flat.device)).to(torch.int32)
    return order, place, offsets


def _scale(span, steps):
    """span / steps (64 bits) rounded once to bfloat16's 8 bits, ties to even.  A division by a Python number would be a product with its
    fp32 reciprocal on the GPU, and .to(bfloat16) from 64 bits rounds to 32 bits in between; both are off where the quotient is next to a tie."""
    bits = (span / torch.full_like(span, steps)).view(torch.int64)
    bits = (bits + ((1 << 44) - 1) + (bits >> 45 & 1)) & -(1 << 45)                     # 52 - 7 bits go
    return bits.view(torch.float64).to(torch.bfloat16)


def _quantize(w, group, zero):
    """w [E][N][K] of any type -> whole numbers 0..15 float32 [E][N][Kp], scale bf16 and zero float32 [E][N][groups]; K padded to 128."""
    E, N, K = w.shape
    Kp = -(-K // 128) * 128
    g = torch.nn.functional.pad(w.float(), (0, Kp - K)).reshape(E, N, Kp // group, group)
    if zero:
        lo, hi = g.amin(3).clamp(max=0), g.amax(3).clamp(min=0)
        scale = _scale(hi.double() - lo.double(), 15.0)
        s = scale.float()
        z = torch.where(s > 0, (-lo / s).round(), 0.0).clamp(0, 15)
        q = torch.where(s[..., None] > 0, (g / s[..., None]).round(), 0.0)
    else:
        scale = _scale(g.abs().amax(3).double(), 7.0)
        s = scale.float()
        z = torch.full_like(s, 8.0)
        q = torch.where(s[..., None] > 0, (g / s[..., None]).round(), 0.0)
    q = (q + z[..., None]).clamp(0, 15)
    return q.reshape(E, N, Kp), scale, z


def _piece(device):
    """Position of quarter t in row r of a tile (its own inverse): [128][4]."""
    r = torch.arange(128, device=device)
    return torch.arange(4, device=device)[None, :] ^ ((r[:, None] >> 1) & 3)


def _pack(q, scale, z, zero):
    """Whole numbers, scales and zeros of _quantize -> the stored tiles."""
    E, N, Kp = q.shape
    Np = -(-N // 128) * 128
    v = torch.nn.functional.pad(q.to(torch.uint8), (0, 0, 0, Np - N), value=8)
    v = v.reshape(E, Np // 128, 128, Kp // 128, 4, 4, 8)                                # e, tile, r, ktile, b, t, i
    by = v[..., [0, 4, 1, 5]] | (v[..., [2, 6, 3, 7]] << 4)
    by = by.permute(0, 1, 3, 2, 5, 4, 6).contiguous()                                  # e, tile, ktile, r, t, b, byte
    at = _piece(q.device)[None, None, None, :, :, None, None].expand_as(by)
    by = torch.gather(by, 4, at)
    pad = lambda t, val: torch.nn.functional.pad(t.transpose(1, 2), (0, Np - N), value=val).contiguous()
    return by.reshape(E, Np // 128, Kp // 128, 128, 64), pad(scale, 0.0), pad(z.to(torch.uint8), 8) if zero else None


def _unpack(q, scale, zero, N, K, group):
    """The stored tiles -> float32 weights [E][N][K]."""
    E, nt, kt = q.shape[:3]
    by = q.reshape(E, nt, kt, 128, 4, 4, 4)
    at = _piece(q.device)[None, None, None, :, :, None, None].expand_as(by)
    by = torch.gather(by, 4, at)
    lo, hi = by & 15, by >> 4
    v = torch.stack([lo[..., 0], lo[..., 2], hi[..., 0], hi[..., 2], lo[..., 1], lo[..., 3], hi[..., 1], hi[..., 3]], dim=-1)
    v = v.permute(0, 1, 3, 2, 5, 4, 6).reshape(E, nt * 128, kt * 128 // group, group).float()
    v -= 8.0 if zero is None else zero.transpose(1, 2)[..., None].float()
    v *= scale.transpose(1, 2)[..., None].float()
    return v.reshape(E, nt * 128, kt * 128)[:, :N, :K]


def _uneven(gen, rows, E, active):
    """Rows of each expert (a list of E counts): `active` of them have some, unevenly."""
    who = torch.randperm(E, device="cuda", generator=gen)[:active]
    share = torch.rand(active, device="cuda", generator=gen) + 0.25
    extra = torch.multinomial(share, rows - active, replacement=True, generator=gen) if rows > active else who[:0]
    count = torch.zeros(E, dtype=torch.int64, device="cuda")
    count[who] = 1 + torch.bincount(extra, minlength=active)
    return count


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)
    op = case["op"]
    s = dict(case=case)
    if op == "route":
        s["expert"] = _experts(gen, case["n"], case["k"], case["E"], case["left_out"])
        return s
    if op == "move":
        n, k, D, dt = case["n"], case["k"], case["D"], DTYPE[case["dtype"]]
        expert = _experts(gen, n, k, 32, case["left_out"])
        _, s["place"], s["offsets"] = _plain_route(expert, 32)
        s["x"] = rnd(n, D).to(dt)
        s["w"] = torch.softmax(rnd(n, k), dim=1)
        s["ye"] = rnd(n * k, D).to(dt)                                                  # what the experts answered, in sorted order
        if case["train"]:
            s["dout"] = rnd(n, D).to(dt)
            s["dxs"] = rnd(n * k, D).to(dt)                                             # gradient of the dispatched rows
        return s
    N, K, group = case["N"], case["K"], case["group"]
    E = case.get("E", 1)
    w = rnd(E, N, K) / math.sqrt(K)
    if op == "quantize":
        s["weight"] = w.to(DTYPE[case["dtype"]])
        return s
    s["q"], s["scale"], s["zero"] = _pack(*_quantize(w, group, case["zero"]), case["zero"])
    del w
    s["x"] = rnd(case["rows"], K).to(DTYPE[case["dtype"]])
    s["bias"] = 0.1 * rnd(E, N) if case["bias"] else None
    s["offsets"] = s["cap"] = None
    if op == "experts":
        count = _uneven(gen, case["rows"], E, case["active"])
        s["offsets"] = torch.nn.functional.pad(count.cumsum(0), (1, 0)).to(torch.int32)
        # the plain form's batched product: the most rows of an expert, the experts that have rows and each expert's number among them
        s["cap"], s["who"], s["nth"] = int(count.max()), torch.nonzero(count)[:, 0], (count > 0).cumsum(0) - 1
    return s


# ---------------------------------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    bls = _lib()
    c = s["case"]
    op = c["op"]
    new = lambda like, *shape, dtype=None: torch.empty(shape, dtype=dtype or like.dtype, device=like.device)
    if op == "route":
        e = s["expert"]
        n, k = e.shape
        order, place, offsets = new(e, n * k), new(e, n, k), new(e, c["E"] + 1)
        bls.bls_moe_route(e, c["E"], order, place, offsets)
        return dict(order=order, place=place, offsets=offsets)
    if op == "move":
        x, ye, w, place, offsets = s["x"], s["ye"], s["w"], s["place"], s["offsets"]
        xs, out = torch.empty_like(ye), torch.empty_like(x)
        bls.bls_moe_dispatch(x, place, offsets, xs)
        bls.bls_moe_combine(ye, place, w, out)
        if not c["train"]:
            return dict(xs=xs, out=out)
        dye, dw, dx = torch.empty_like(ye), torch.empty_like(w), torch.empty_like(x)
        bls.bls_moe_combine_grad(s["dout"], ye, place, offsets, w, dye, dw)
        bls.bls_moe_combine(s["dxs"], place, None, dx)
        return dict(xs=xs, out=out, dye=dye, dw=dw, dx=dx)
    if op == "quantize":
        w4 = bls.bls_w4_quantize(s["weight"], c["group"], not c["zero"])
        w = torch.empty_like(s["weight"])
        bls.bls_w4_dequantize(w4, w)
        return dict(w=w, scale=w4.scale)
    w4 = bls.W4(s["q"], s["scale"], s["zero"], c["N"], c["K"], c["group"])
    y = new(s["x"], c["rows"], c["N"])
    bls.bls_w4_linear(w4, s["x"], y, offsets=s["offsets"], bias=s["bias"], act=c["act"])
    return dict(y=y)


def _plain_combine(y, place, w):
    here = place >= 0
    g = y[place.clamp(min=0).long()].float()                                            # [n][k][D]
    g = torch.where(here[..., None], g, 0.0)
    return (g if w is None else g * w[..., None]).sum(1)


def _plain_spread(rows, place, total_rows):
    """rows [n][k][D] float32 -> [total_rows][D], each at its place, zeros elsewhere."""
    D = rows.shape[2]
    out = torch.zeros(total_rows + 1, D, dtype=rows.dtype, device=rows.device)          # the last row takes what has no place
    out[torch.where(place >= 0, place.long(), total_rows).reshape(-1)] = rows.reshape(-1, D)
    return out[:total_rows]


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "route":
        order, place, offsets = _plain_route(s["expert"], c["E"])
        return dict(order=order, place=place, offsets=offsets)
    if op == "move":
        x, ye, w, place = s["x"], s["ye"], s["w"], s["place"]
        n, k = place.shape
        dt = x.dtype
        xs = _plain_spread(x.float()[:, None, :].expand(n, k, x.shape[1]), place, n * k).to(dt)
        out = _plain_combine(ye, place, w).to(dt)
        if not c["train"]:
            return dict(xs=xs, out=out)
        dout = s["dout"].float()
        dye = _plain_spread(w[..., None] * dout[:, None, :], place, n * k).to(dt)
        g = ye[place.clamp(min=0).long()].float()
        dw = torch.where(place >= 0, (g * dout[:, None, :]).sum(2), 0.0)
        return dict(xs=xs, out=out, dye=dye, dw=dw, dx=_plain_combine(s["dxs"], place, None).to(dt))
    N, K, group = c["N"], c["K"], c["group"]
    if op == "quantize":
        q, scale, z = _quantize(s["weight"], group, c["zero"])
        v = (q.reshape(*z.shape, group) - z[..., None]) * scale.float()[..., None]
        pad = -N % 128                                                                  # scales are stored by group, rows padded to 128
        return dict(w=v.reshape(q.shape)[:, :, :K].to(s["weight"].dtype),
                    scale=torch.nn.functional.pad(scale.transpose(1, 2), (0, pad)).contiguous())
    x, bias, off = s["x"].float(), s["bias"], s["offsets"]
    if off is None:
        y = x @ _unpack(s["q"], s["scale"], s["zero"], N, K, group)[0].t()
        if bias is not None:
            y = y + bias[0]
    else:
        who, cap = s["who"], s["cap"]
        w = _unpack(s["q"][who], s["scale"][who], None if s["zero"] is None else s["zero"][who], N, K, group)
        at = torch.arange(x.shape[0], device=x.device)
        e = (at[:, None] >= off[None, 1:]).sum(1)                                       # expert of a row
        i = at - off[e]
        xp = torch.zeros(who.numel(), cap, K, device=x.device)
        xp[s["nth"][e], i] = x
        y = torch.bmm(xp, w.transpose(1, 2))[s["nth"][e], i]
        if bias is not None:
            y = y + bias[e]
    y = torch.relu(y) if c["act"] == 1 else torch.sigmoid(y) if c["act"] == 2 else y
    return dict(y=y.to(s["x"].dtype))


# ---------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "route":
        return dict(bytes=12 * case["n"] * case["k"] + 4 * (case["E"] + 1), flops=0)
    if op == "move":
        n, k, D = case["n"], case["k"], case["D"]
        b = 4 if case["dtype"] == "f32" else 2
        rows = n * k
        lists = 8 * rows                                                                # places and weights
        kept = rows * (1.0 - case["left_out"])                                          # rows of the experts that are read
        total = (n * D + rows * D + kept * D + n * D) * b + lists
        flops = 2.0 * kept * D
        if case["train"]:
            total += (n * D + rows * D + kept * D + n * D) * b + 4 * rows
            flops += 4.0 * kept * D
        return dict(bytes=total, flops=flops)
    N, K = case["N"], case["K"]
    groups = -(-K // case["group"])
    if op == "quantize":
        b = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=case["E"] * N * (2.0 * K * b + groups * 2), flops=4.0 * case["E"] * N * K)
    used = case.get("active", 1)
    rows = case["rows"]
    weights = used * N * (K / 2 + groups * (3 if case["zero"] else 2)) + (4 * used * N if case["bias"] else 0)
    return dict(bytes=weights + 2.0 * rows * (K + N), flops=2.0 * rows * N * K)


# ---------------------------------------------------------------------------------------- 64 bits, from the definition

def _exact_weights(s, e, N, K, group):
    """Expert e's weights in 64 bits: every element's byte is found by its own address."""
    q = s["q"][e].reshape(-1)
    kt = s["q"].shape[2]
    n = torch.arange(N, device=q.device)[:, None]
    k = torch.arange(K, device=q.device)[None, :]
    i = k % 8
    where = ((n // 128) * kt + k // 128) * 8192 + (n % 128) * 64
    where = where + ((((k % 128) // 8) % 4) ^ ((n % 128) // 2 % 4)) * 16 + ((k % 128) // 32) * 4
    where = where + (i % 2) * 2 + i // 4
    v = (q[where] >> (4 * ((i // 2) % 2)).to(torch.uint8)) & 15
    z = 8.0 if s["zero"] is None else s["zero"][e].double()[(k // group)[0], :N].t()
    return (v.double() - z) * s["scale"][e].double()[(k // group)[0], :N].t()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        return None                                                                     # whole numbers only
    if op == "move":
        n, k = s["place"].shape
        D = case["D"]
        slot = torch.nonzero(s["place"].reshape(-1) >= 0)[:, 0]                        # the slots that have a place
        place, token = s["place"].reshape(-1).long()[slot], slot // k
        wt = s["w"].reshape(-1).double()[slot, None]

        def rows(src):                                                                  # a row for each place
            o = torch.zeros(n * k, D, dtype=torch.float64, device="cuda")
            o[place] = src
            return o

        def sums(y, weight):                                                            # a sum for each token
            o = torch.zeros(n, D, dtype=torch.float64, device="cuda")
            return o.index_add_(0, token, y.double()[place] * weight)

        r = dict(xs=rows(s["x"].double()[token]), out=sums(s["ye"], wt))
        if case["train"]:
            d = s["dout"].double()
            r["dye"] = rows(wt * d[token])
            dw = torch.zeros(n * k, dtype=torch.float64, device="cuda")
            dw[slot] = torch.einsum("rd,rd->r", s["ye"].double()[place], d[token])
            r["dw"] = dw.reshape(n, k)
            r["dx"] = sums(s["dxs"], 1.0)
        return r
    N, K, group = case["N"], case["K"], case["group"]
    if op == "quantize":
        w = s["weight"].double()
        E, Np, Kp = w.shape[0], -(-N // 128) * 128, -(-K // 128) * 128
        full = torch.zeros(E, Np, Kp, dtype=torch.float64, device="cuda")
        full[:, :N, :K] = w
        full = full.reshape(E, Np, -1, group)
        if case["zero"]:
            lo = torch.minimum(full.min(3).values, torch.zeros((), device="cuda", dtype=torch.float64))
            hi = torch.maximum(full.max(3).values, torch.zeros((), device="cuda", dtype=torch.float64))
            scale = ((hi - lo) / 15).to(torch.bfloat16).double()                        # the scale is held in bfloat16 by definition
            least = 0
        else:
            lo = torch.zeros((), device="cuda", dtype=torch.float64)
            scale = (full.abs().max(3).values / 7).to(torch.bfloat16).double()
            least = -8
        safe = torch.where(scale > 0, scale, 1.0)
        shift = torch.round(-lo / safe).clamp(0, 15)
        step = torch.round(full / safe[..., None]) + shift[..., None]
        step = step.clamp(least, least + 15) - shift[..., None]
        return dict(w=(step * scale[..., None]).reshape(E, Np, Kp)[:, :N, :K], scale=scale.transpose(1, 2))
    x = s["x"].double()
    ends = [0, case["rows"]] if s["offsets"] is None else s["offsets"].tolist()
    y = torch.empty(case["rows"], N, dtype=torch.float64, device="cuda")
    for e in range(len(ends) - 1):
        a, b = ends[e], ends[e + 1]
        if a < b:
            y[a:b] = x[a:b] @ _exact_weights(s, e, N, K, group).t()
            if s["bias"] is not None:
                y[a:b] += s["bias"][e].double()
    y = y.clamp(min=0) if case["act"] == 1 else 1 / (1 + torch.exp(-y)) if case["act"] == 2 else y
    return dict(y=y)
