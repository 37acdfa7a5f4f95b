"""The 8-bit cache, measured: tokens quantised as they are written and read back, and attention over the cache.

A cache holds keys and values in 8 bits (int8 or e4m3), one power-of-two scale for every block of 16 tokens of a KV
head.  Each case below is a call that serving with Cartridges makes of it: appending a step's tokens, storing a message
or a whole context, one decode step over private, shared or composed Cartridges, attention of a new message's tokens.

    listed()            the cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs on the GPU, and the handles that a serving program holds
    run(state)          one pass: plain torch operations, or (own) the library's calls
    exact(case, seed)   the same outputs from the definitions, in 64 bits
    work(case)          the bytes and operations that a pass cannot do without
"""
import math
import random

import numpy as np
import torch

own = False

D = 128          # head dimension
BLOCK = 16       # tokens that share a scale
E_MIN = -120     # smallest scale exponent
LARGEST = {"int8": 127.0, "e4m3": 448.0}


# ---- cases -----------------------------------------------------------------------------------------------------------

def _case(name, op, fmt, hq, hkv, batch, prefix="none", p=0, members=0, lo=0, hi=0, new_lo=1, new_hi=1):
    """op: "store" (write, then read back), "attend" (the last new_lo .. new_hi tokens of every cache ask), "step" (write
    one token, attend, read the block it went to).  prefix: whose Cartridges of p tokens stand before a request's own
    tokens: "none", "private" (one each), "shared" (one for all), "pool" (two out of `members`).  lo .. hi: own tokens,
    before the write (store, step) or in all (attend)."""
    return dict(name=name, op=op, fmt=fmt, hq=hq, hkv=hkv, batch=batch, prefix=prefix, p=p, members=members, lo=lo, hi=hi,
                new_lo=new_lo, new_hi=new_hi)


def listed():
    return [
        # one decode step's tokens of 64 conversations join their caches, most of them inside a block
        _case("store a step, 64 requests", "store", "int8", 24, 8, 64, lo=1, hi=512),
        # the messages of seven users, of very unequal lengths, behind what they have
        _case("store 7 messages", "store", "e4m3", 32, 8, 7, lo=0, hi=300, new_lo=1, new_hi=1500),
        # a full context of 100 k tokens is taken over into 8 bits
        _case("store a 100k context", "store", "int8", 32, 8, 1, new_lo=100000, new_hi=100000),
        # the first token of a conversation without a Cartridge: a cache of one token
        _case("attend, one token", "attend", "e4m3", 8, 8, 1, lo=1, hi=1),
        # a small batch over short Cartridges: latency
        _case("attend, 4 x (512 + 64)", "attend", "int8", 24, 8, 4, "private", 512, lo=64, hi=64),
        # 64 users, each with a Cartridge: the decode step of the benchmark's headline
        _case("attend, 64 x (2048 + 1..512)", "attend", "int8", 24, 8, 64, "private", 2048, lo=1, hi=512),
        # one Cartridge for 128 users
        _case("attend, 128 share 4096", "attend", "e4m3", 32, 8, 128, "shared", 4096, lo=1, hi=1024),
        # full contexts instead of Cartridges
        _case("attend, 8 x 100k", "attend", "int8", 32, 8, 8, lo=100000, hi=100000),
        # one long conversation, eight heads to a KV head, an odd length
        _case("attend, 1 x 131071", "attend", "e4m3", 64, 8, 1, lo=131071, hi=131071),
        # composed Cartridges, the token written and attended to in one call
        _case("step, 96 x (2 of 16 x 2048)", "step", "int8", 32, 8, 96, "pool", 2048, 16, lo=1, hi=512),
        # a user's message over a Cartridge
        _case("attend, message 512 on 2048", "attend", "e4m3", 24, 8, 1, "private", 2048, lo=512, hi=512, new_lo=512, new_hi=512),
        # messages of several users in one call, next to users that decode, over a Cartridge of an odd length
        _case("attend, 6 ragged messages", "attend", "int8", 32, 8, 6, "shared", 1999, lo=900, hi=6000, new_lo=1, new_hi=900),
    ]


def _between(rng, lo, hi):
    """A whole number of lo .. hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["store", "attend", "attend", "step", "message"])
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
        fmt = rng.choice(["int8", "e4m3"])
        prefix, p, members, new_lo, new_hi = "none", 0, 0, 1, 1
        if op == "store":
            batch = _between(rng, 1, 128)
            lo = rng.choice([0, 1, 15, 16, 17, 100])
            hi = lo + _between(rng, 1, 500)
            new_hi = _between(rng, 1, 100000 // batch)
            new_lo = rng.choice([1, new_hi, max(1, new_hi // 3)])
        elif op == "message":
            op = "attend"
            batch = _between(rng, 1, 8)
            new_hi = _between(rng, 2, 1000)
            new_lo = rng.choice([1, new_hi])
            lo, hi = new_hi, new_hi + _between(rng, 1, 5000)
        else:
            batch = _between(rng, 1, 128)
            lo = _between(rng, 1, 100)
            hi = max(lo, _between(rng, 1, 100000 // batch))
        if op != "store":
            prefix = rng.choice(["none", "private", "shared", "pool"])
            if prefix != "none":
                p = _between(rng, 1, 4096)
            if prefix == "pool":
                members = rng.randint(2, 16)
        c = _case("", op, fmt, hq, hkv, batch, prefix, p, members, lo, hi, new_lo, new_hi)
        del c["name"]
        w = work(c)
        if w["bytes"] <= 1.6e9 and w["flops"] <= 2.5e11:
            return c


def _batch(case):
    """What the case's numbers say: for every request the caches before it, its own tokens and how many are new; the
    lengths of the Cartridges.  A function of the case alone."""
    rng = random.Random("%(op)s %(batch)d %(prefix)s %(p)d %(members)d %(lo)d %(hi)d %(new_lo)d %(new_hi)d" % case)
    n = case["batch"]
    own_len = [rng.randint(case["lo"], case["hi"]) for _ in range(n)]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
    if case["op"] == "attend":
        new = [min(a, b) for a, b in zip(new, own_len)]
    else:
        own_len = [a + b for a, b in zip(own_len, new)]
    n_parts = {"none": 0, "private": n, "shared": 1, "pool": case["members"]}[case["prefix"]]
    parts = [[], ] * n if not n_parts else [
        {"private": lambda i: [i], "shared": lambda i: [0], "pool": lambda i: rng.sample(range(n_parts), 2)}[case["prefix"]](i)
        for i in range(n)]
    return own_len, new, parts, [case["p"]] * n_parts


def work(case):
    own_len, new, parts, part_len = _batch(case)
    hq, hkv = case["hq"], case["hkv"]
    token = 2 * hkv * D                                        # K and V of a token, 8 bits each
    scales = 2 * hkv / BLOCK
    if case["op"] == "store":
        n = sum(new)
        return {"bytes": int(n * (2 * 2 * token + 2 * (token + scales))), "flops": 4 * n * token}
    held = sum(own_len) + sum(part_len[j] for j in set(sum(parts, [])))
    keys = sum(sum(part_len[j] for j in q) * m + m * (a - m) + m * (m + 1) // 2 for a, m, q in zip(own_len, new, parts))
    rows = sum(new)
    n_bytes = held * (token + scales) + rows * hq * (2 * 2 * D + 4)
    if case["op"] == "step":
        n_bytes += len(new) * 2 * token + sum((a - 1) % BLOCK + 1 for a in own_len) * 2 * token   # the new rows; the block read back
    return {"bytes": int(n_bytes), "flops": 4 * hq * D * keys}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _normal(shape, gen, outliers=False):
    """N(0, 1) in bf16; outliers: one key channel in 250 is eight times as large, as trained keys' channels are."""
    x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
    for a in range(0, shape[0], 1 << 17):
        x[a:a + (1 << 17)] = torch.randn((min(1 << 17, shape[0] - a),) + tuple(shape[1:]), generator=gen, device="cuda")
    if outliers:
        x *= torch.where(torch.rand(shape[1:], generator=gen, device="cuda") < 0.004, 8.0, 1.0).to(torch.bfloat16)
    return x


def _inputs(case, seed):
    """Keys and values of every cache, cache after cache on one token axis (Cartridges first), and the queries."""
    own_len, new, parts, part_len = _batch(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens = part_len + own_len
    n = sum(lens)
    k = _normal((n, case["hkv"], D), gen, True)
    v = _normal((n, case["hkv"], D), gen)
    q = _normal((sum(new), case["hq"], D), gen) * 2 if case["op"] != "store" else None
    return lens, k, v, q


def _ints(values):
    return torch.tensor(values, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    own_len, new, parts, part_len = _batch(case)
    lens, k, v, q = _inputs(case, seed)
    n_parts, n = len(part_len), len(own_len)
    at = np.concatenate([[0], np.cumsum(lens)]).astype(int)
    op, hkv = case["op"], case["hkv"]
    state = {"case": case, "q": q}
    first = [a - m for a, m in zip(own_len, new)]                     # where a write begins
    back = [f // BLOCK * BLOCK for f in first]                        # where reading back begins
    if op != "attend":
        rows = _ints(np.concatenate([np.arange(at[n_parts + i] + first[i], at[n_parts + i + 1]) for i in range(n)]))
        state["k_new"], state["v_new"] = k[rows], v[rows]
    if own:
        from paper_2506_06266_b200 import binding, buildlib
        buildlib.build()
        cfg = binding.make_config(1, case["hq"], hkv, max(sum(new) if op == "attend" else n, 1), 1, max_parts=2)
        room = binding.cart_scratch_bytes(cfg) + binding.cart_q8_scratch_bytes(cfg)
        room += sum(binding.cart_q8_cache_bytes(cfg, t) for t in lens)
        arena = torch.empty(room + 4096, dtype=torch.uint8, device="cuda")
        cfg.arena, cfg.arena_bytes = arena.data_ptr(), arena.numel()
        ctx = binding.cart_create(cfg)
        fmt = {"int8": binding.CART_Q8_INT8, "e4m3": binding.CART_Q8_E4M3}[case["fmt"]]
        here = torch.cuda.current_stream()
        ids = []
        for i, t in enumerate(part_len + (own_len if op == "attend" else first)):   # a Cartridge is written before it is a part
            mine = [] if i < n_parts else [ids[j] for j in parts[i - n_parts]]
            ids.append(binding.cart_q8_open(ctx, fmt, mine, lens[i]))
            if t:
                binding.cart_q8_write(ctx, 0, [ids[i]], [t], k[at[i]:at[i] + t], v[at[i]:at[i] + t], stream=here)
        state |= {"b": binding, "ctx": _Context(binding, ctx, arena), "ids": binding.ReqList(ids[n_parts:])}
        state |= {"first": binding.ReqList(first), "new": binding.ReqList(new), "back": binding.ReqList(back)}
        state["n_back"] = binding.ReqList([a - b for a, b in zip(own_len, back)])
        if op != "attend":
            state["k_back"] = torch.empty((sum(own_len) - sum(back), hkv, D), dtype=torch.bfloat16, device="cuda")
            state["v_back"] = torch.empty_like(state["k_back"])
        if q is not None:
            state["out"] = torch.empty_like(q)
            state["lse"] = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
        torch.cuda.synchronize()
        return state
    # Plain: every cache padded to whole blocks on one axis of blocks
    blocks = [(t + BLOCK - 1) // BLOCK for t in lens]
    b0 = np.concatenate([[0], np.cumsum(blocks)]).astype(int)
    token = np.concatenate([b0[i] * BLOCK + np.arange(t) for i, t in enumerate(lens)] + [np.zeros(0, int)])
    written = np.zeros(b0[-1] * BLOCK, bool)                          # held before the pass
    for i, t in enumerate(part_len + (own_len if op == "attend" else first)):
        written[b0[i] * BLOCK:b0[i] * BLOCK + t] = True
    token, written = _ints(token), torch.from_numpy(written).cuda()
    for name, x in (("k", k), ("v", v)):
        padded = torch.zeros((b0[-1] * BLOCK, hkv, D), dtype=torch.bfloat16, device="cuda")
        padded[token] = x
        padded[~written] = 0
        state[name + "_codes"], state[name + "_exp"] = _quantise(padded.view(-1, BLOCK, hkv, D), case["fmt"])
    if op != "attend":
        put = [b0[n_parts + i] * BLOCK + np.arange(first[i], own_len[i]) for i in range(n)]
        read = [b0[n_parts + i] * BLOCK + np.arange(back[i], own_len[i]) for i in range(n)]
        state["put"], state["read"] = _ints(np.concatenate(put)), _ints(np.concatenate(read))
        state["held"] = written
    if q is not None:
        total = [a + sum(part_len[j] for j in parts[i]) for i, a in enumerate(own_len)]
        keys = np.zeros((n, max(total)), int)                         # where request i's key j lies
        for i in range(n):
            where = [b0[j] * BLOCK + np.arange(part_len[j]) for j in parts[i]]
            where.append(b0[n_parts + i] * BLOCK + np.arange(own_len[i]))
            keys[i, :total[i]] = np.concatenate(where)
        ask = np.full((n, max(new)), sum(new))                        # where request i's query r lies (one behind the last: nowhere)
        for i, r0 in enumerate(np.concatenate([[0], np.cumsum(new)[:-1]]).astype(int)):
            ask[i, :new[i]] = r0 + np.arange(new[i])
        sees = np.zeros((n, max(new)), int)                           # how many keys it sees
        for i in range(n):
            sees[i, :new[i]] = total[i] - new[i] + 1 + np.arange(new[i])
        state |= {"keys": _ints(keys), "ask": _ints(ask), "sees": _ints(sees)}
    return state


class _Context:
    """A library context that lives as long as the state that holds it."""

    def __init__(self, binding, ctx, arena):
        self.binding, self.ctx, self.arena = binding, ctx, arena

    def __del__(self):
        self.binding.cart_destroy(self.ctx)


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _exponent(largest, fmt):
    """The smallest exponent e with largest <= LARGEST * 2^e."""
    m, e = torch.frexp(largest.float())                               # largest = m * 2^e, 0.5 <= m < 1
    e = e.to(torch.int32)
    e = torch.where(m <= 127 / 128, e - 7, e - 6) if fmt == "int8" else torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(largest > 0, e, E_MIN).clamp_min(E_MIN)


def _round(x, fmt):
    """The nearest value that a code has, ties to even."""
    return torch.round(x) if fmt == "int8" else x.to(torch.float8_e4m3fn).float()


def _codes(x, e, fmt):
    return _round(torch.ldexp(x.float(), -e[:, None, :, None]), fmt).to(torch.int8 if fmt == "int8" else torch.float8_e4m3fn)


def _quantise(x, fmt):
    """x [blocks][16][heads][128] -> codes of the same shape, exponents [blocks][heads]."""
    e = _exponent(x.abs().amax(dim=(1, 3)), fmt)
    codes = torch.empty(x.shape, dtype=torch.int8 if fmt == "int8" else torch.float8_e4m3fn, device=x.device)
    for a in range(0, x.shape[0], 1 << 14):
        codes[a:a + (1 << 14)] = _codes(x[a:a + (1 << 14)], e[a:a + (1 << 14)], fmt)
    return codes, e


def _values(codes, e):
    return torch.ldexp(codes.float(), e[:, None, :, None])


def _store(state, name):
    """The tokens behind a block's held ones are quantised with them: the scale grows to what the largest needs, and codes
    that are held already are rounded once more to the grown scale."""
    fmt = state["case"]["fmt"]
    codes, e_old = state[name + "_codes"], state[name + "_exp"]
    fresh = torch.zeros(codes.shape, dtype=torch.bfloat16, device=codes.device)
    fresh.view(-1, *codes.shape[2:])[state["put"]] = state[name + "_new"]
    e = _exponent(fresh.abs().amax(dim=(1, 3)), fmt)
    begun = state["held"].view(-1, BLOCK)[:, 0]                       # blocks that hold something have a scale
    e = torch.where(begun[:, None], torch.maximum(e, e_old), e)
    kept = _round(torch.ldexp(codes.float(), (e_old - e)[:, None, :, None]), fmt)
    now = torch.where(state["held"].view(-1, BLOCK)[:, :, None, None], kept, _codes(fresh, e, fmt).float())
    return now, e


def _attend(state, k, v):
    """Softmax attention of every request's queries over the tokens that they see; k and v [tokens][heads][128], fp32."""
    case = state["case"]
    hq, hkv = case["hq"], case["hkv"]
    ask, sees, keys = state["ask"], state["sees"], state["keys"]
    n, m = ask.shape
    q = torch.cat([state["q"].float(), torch.zeros((1, hq, D), device="cuda")])[ask]        # [n][m][hq][D]
    q = q.view(n, m, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, D)
    s = torch.matmul(q, k[keys].permute(0, 2, 3, 1)) * D ** -0.5                            # [n][hkv][G m][keys]
    s = s.view(n, hkv, hq // hkv, m, -1)
    unseen = torch.arange(s.shape[-1], device="cuda") >= sees[:, None, None, :, None]
    s = s.masked_fill(unseen, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    s = torch.exp(s - top)
    total = s.sum(-1, keepdim=True)
    out = torch.matmul(s.view(n, hkv, -1, s.shape[-1]), v[keys].permute(0, 2, 1, 3)).view(n, hkv, -1, m, D) / total
    lse = (torch.log(total) + top).squeeze(-1)
    asked = ask < state["q"].shape[0]
    out = out.permute(0, 3, 1, 2, 4).reshape(n, m, hq, D)[asked]
    return out.to(torch.bfloat16), lse.permute(0, 3, 1, 2).reshape(n, m, hq)[asked]


def run(state):
    op = state["case"]["op"]
    if own:
        b, ctx, ids, here = state["b"], state["ctx"].ctx, state["ids"], torch.cuda.current_stream()
        if op == "store":
            b.cart_q8_write(ctx, 0, ids, state["new"], state["k_new"], state["v_new"], first=state["first"], stream=here)
        elif op == "attend":
            b.cart_q8_attention(ctx, 0, ids, state["q"], state["out"], state["lse"], n_new=state["new"], stream=here)
        else:
            b.cart_q8_decode_step(ctx, 0, ids, state["k_new"], state["v_new"], state["q"], state["out"], state["lse"],
                                  first=state["first"], stream=here)
        if op != "attend":
            b.cart_q8_read(ctx, 0, ids, state["back"], state["n_back"], state["k_back"], state["v_back"], stream=here)
        return {x: state[x] for x in ("k_back", "v_back", "out", "lse") if x in state}
    got = {}
    if op == "attend":
        k, v = (_values(state[x + "_codes"], state[x + "_exp"]).flatten(0, 1) for x in "kv")
    else:
        k, v = (_values(*_store(state, x)).flatten(0, 1) for x in "kv")
        got["k_back"], got["v_back"] = (x[state["read"]].to(torch.bfloat16) for x in (k, v))
    if op != "store":
        got["out"], got["lse"] = _attend(state, k, v)
    return got


# ---- the definitions, in 64 bits -------------------------------------------------------------------------------------

def _grid(x, fmt):
    """x (float64) on the grid of the format's values: half to even."""
    if fmt == "int8":
        return torch.round(x)
    # three mantissa bits; below 2^-6 the steps stay 2^-9
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _held(x, n_held, fmt):
    """What a cache stands for after its first n_held tokens were written at once and the others after them: x [n][heads][128]
    in float64."""
    out = torch.empty_like(x)
    top = LARGEST[fmt]
    for a, b in ((0, n_held // BLOCK * BLOCK), (n_held // BLOCK * BLOCK, x.shape[0])):
        if a == b:
            continue
        pad = torch.zeros(((-(b - a)) % BLOCK,) + x.shape[1:], dtype=x.dtype, device=x.device)
        y = torch.cat([x[a:b], pad]).view(-1, BLOCK, *x.shape[1:])

        def scale(z):
            big = z.abs().amax(dim=(1, 3), keepdim=True)
            e = torch.ceil(torch.log2(big / top))
            e = torch.where(top * torch.exp2(e - 1) >= big, e - 1, torch.where(top * torch.exp2(e) < big, e + 1, e))
            return torch.exp2(e.clamp_min(E_MIN))
        if a == 0 and b <= n_held:
            s = scale(y)
            z = _grid(y / s, fmt) * s
        else:
            early = y.clone().flatten(0, 1)
            early[n_held - a:] = 0
            late = y.clone().flatten(0, 1)
            late[:n_held - a] = 0
            early, late = early.view_as(y), late.view_as(y)
            s0 = scale(early)
            s = torch.maximum(s0, scale(late))
            z = _grid(_grid(early / s0, fmt) * s0 / s, fmt) * s + _grid(late / s, fmt) * s
        out[a:b] = z.flatten(0, 1)[:b - a]
    return out


def exact(case, seed):
    own_len, new, parts, part_len = _batch(case)
    lens, k, v, q = _inputs(case, seed)
    at = np.concatenate([[0], np.cumsum(lens)]).astype(int)
    n_parts, hkv, g = len(part_len), case["hkv"], case["hq"] // case["hkv"]
    held = part_len + (own_len if case["op"] == "attend" else [a - m for a, m in zip(own_len, new)])

    def cache(j):
        return [_held(x[at[j]:at[j + 1]].double(), held[j], case["fmt"]) for x in (k, v)]
    z = [cache(j) for j in range(n_parts)]
    got, r0 = {"k_back": [], "v_back": [], "out": [], "lse": []}, 0
    for i, m in enumerate(new):
        mine = cache(n_parts + i)
        if case["op"] != "attend":
            a = held[n_parts + i] // BLOCK * BLOCK
            got["k_back"].append(mine[0][a:])
            got["v_back"].append(mine[1][a:])
        if q is None:
            continue
        ki, vi = (torch.cat([z[j][x] for j in parts[i]] + [mine[x]]) for x in (0, 1))
        out, lse = (torch.empty((m, hkv, g) + t, dtype=torch.float64, device="cuda") for t in ((D,), ()))
        sees = ki.shape[0] - m + 1 + torch.arange(m, device="cuda")
        for h in range(hkv):
            s = torch.einsum("mgd,nd->mgn", q[r0:r0 + m].double().view(m, hkv, g, D)[:, h], ki[:, h]) / math.sqrt(D)
            s[(torch.arange(ki.shape[0], device="cuda") >= sees[:, None])[:, None, :].expand_as(s)] = -math.inf
            lse[:, h] = torch.logsumexp(s, -1)
            out[:, h] = torch.einsum("mgn,nd->mgd", torch.exp(s - lse[:, h, :, None]), vi[:, h])
        got["out"].append(out.reshape(m, hkv * g, D))
        got["lse"].append(lse.reshape(m, hkv * g))
        r0 += m
    return {x: torch.cat(y) for x, y in got.items() if y}
