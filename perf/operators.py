"""Dense attention beside the sparse operator, as programs use it.

Three operators:

cross    attention of a batch's tokens to an encoder's states, another length
         for each sequence; query heads share key and value heads
cache    keys and values quantised to 8 bits as they are written into a paged
         cache, and read back
attend   the newest tokens of a batch attend to their own cached keys and to a
         long prefix that the whole batch shares

``own`` false: the operators in plain torch, in 32 bits.  ``own`` true: the
framework's calls.
"""
import math

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _case(name, op, heads=8, kv=8, d=64, dtype="f16", **sizes):
    """q, k, own: the shortest and the longest of the batch's lengths."""
    c = dict(op=op, heads=heads, kv=kv, d=d, dtype=dtype)
    for key, v in sizes.items():
        if key in ("q", "k", "own"):
            c[key + "_least"], c[key] = v
        else:
            c[key] = v
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decoder step of a small batch over short encoder states: latency
        _case("cross_token_small", "cross", batch=4, q=(1, 1), k=(301, 700)),
        # one decoder step of a large batch, shared key heads: bytes of K and V
        _case("cross_token_batch", "cross", heads=32, kv=8, d=128, dtype="bf16", batch=64,
              q=(1, 1), k=(1500, 4097)),
        # a training step on a padded batch of sentences
        _case("cross_train_padded", "cross", batch=8, q=(100, 512), k=(200, 1025), train=True,
              padded=True),
        # a long document read by a long output: the matrix units count
        _case("cross_long", "cross", heads=32, kv=8, d=128, dtype="bf16", batch=2,
              q=(4001, 4096), k=(8000, 8191)),
        # training on long pairs, ragged, four query heads to a key head
        _case("cross_long_train", "cross", heads=16, kv=4, d=128, dtype="bf16", batch=2,
              q=(4001, 4095), k=(4000, 4099), train=True),
        # one token of each sequence of a batch enters the cache and is read back
        _case("cache_token", "cache", kv=8, d=128, dtype="bf16", batch=64, new=1, page=64,
              own=(100, 2000)),
        # long prompts enter the cache and are read back for the next layer's form
        _case("cache_prompt", "cache", kv=8, d=128, dtype="bf16", batch=4, new=8192, page=64,
              own=(7000, 9000)),
        # one sequence, one token, a cache of ordinary length: latency
        _case("attend_one", "attend", batch=1, new=1, page=16, own=(4001, 4001), prefix=0),
        # one token for each sequence of a ragged batch, nothing shared
        _case("attend_batch", "attend", heads=32, kv=8, d=128, dtype="bf16", batch=64, new=1,
              page=64, own=(500, 8192), prefix=0),
        # two very long sequences: the key axis has to be split
        _case("attend_long", "attend", heads=32, kv=8, d=128, dtype="bf16", batch=2, new=1,
              page=128, own=(120000, 131072), prefix=0),
        # many short answers behind one long prompt
        _case("attend_prefix", "attend", heads=32, kv=8, d=128, dtype="bf16", batch=128, new=1,
              page=64, own=(30, 700), prefix=16384),
        # a few drafted tokens at once behind a short prompt that ends inside a page
        _case("attend_draft", "attend", heads=16, kv=4, d=64, batch=16, new=5, page=32,
              own=(5, 2000), prefix=1001),
    ]


# operations, bytes and scores of the listed cases that need most of each
_MOST_FLOPS = 4 * 2 * 4050 * 8095 * 32 * 128
_MOST_SCORES = 2 * 4096 * 8191 * 32
_MOST_BYTES = 700 << 20


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("cross", "cross", "cache", "attend", "attend"))
        kv = rng.choice((1, 2, 3, 4, 8))
        sizes = dict(kv=kv, heads=kv * rng.choice((1, 1, 2, 4, 5, 8)),
                     d=rng.choice((32, 64, 64, 96, 128, 128, 256)),
                     dtype=rng.choice(("f16", "bf16")))
        if op == "cross":
            train = rng.random() < 0.5
            q = 1 if not train and rng.random() < 0.5 else _log_int(rng, 2, 4096)
            k = _log_int(rng, 30, 8192)
            sizes.update(batch=_log_int(rng, 1, 64), q=((q + 1) // 2, q), k=((k + 2) // 3, k))
            if train:
                sizes["train"] = True
            if rng.random() < 0.3:
                sizes["padded"] = True
        else:
            sizes.update(batch=_log_int(rng, 1, 128), page=rng.choice((16, 32, 64, 128, 256)))
            if op == "cache":
                n = 1 if rng.random() < 0.4 else _log_int(rng, 2, 8192)
                sizes.update(new=n, own=(max(1, n // 2), n + _log_int(rng, 1, 2000)))
            else:
                n = rng.choice((1, 1, 1, 2, 5, 16))
                top = _log_int(rng, 20, 131072)
                sizes.update(new=n, own=(top // 8, top),
                             prefix=rng.choice((0, 1)) * _log_int(rng, 20, 32768))
        c = _case(None, op, **sizes)
        w = work(c)
        top = c["batch"] * c["heads"] * (c["q"] * c["k"] if op == "cross" else 0)
        if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES and top <= _MOST_SCORES:
            return c


# ---- sizes ------------------------------------------------------------------------

def _lengths(lo, hi, n, turn=0):
    """n lengths from lo to hi, both among them where n > 1, in mixed order."""
    if n == 1:
        return [hi]
    step = next(s for s in (37, 41, 43, 47) if math.gcd(s, n) == 1)
    return [lo + (hi - lo) * ((i * step + turn) % n) // (n - 1) for i in range(n)]


def _sums(x):
    out = [0]
    for v in x:
        out.append(out[-1] + v)
    return out


def _cross_sizes(c):
    """Lengths of every sequence and the first row of each in Q and in K and V:
    one behind the other, or padded to the longest."""
    q = _lengths(c["q_least"], c["q"], c["batch"])
    k = _lengths(c["k_least"], c["k"], c["batch"], 1)
    if c.get("padded"):
        return q, k, [max(q) * i for i in range(c["batch"] + 1)], \
            [max(k) * i for i in range(c["batch"] + 1)]
    return q, k, _sums(q), _sums(k)


def _own_sizes(c):
    return _lengths(c["own_least"], c["own"], c["batch"])


def work(case):
    c = case
    H, kv, d = c["heads"], c["kv"], c["d"]
    if c["op"] == "cross":
        q, k, q_ptr, k_ptr = _cross_sizes(c)
        pairs = sum(a * b for a, b in zip(q, k))
        # Q, K, V in, O and the log-sum-exp out
        nbytes = 2 * sum(q) * H * d + 4 * sum(k) * kv * d + q_ptr[-1] * H * (2 * d + 4)
        flops = 4 * pairs * H * d
        if c.get("train"):
            # dO in, dQ, dK and dV out
            nbytes += 2 * sum(q) * H * d + 2 * q_ptr[-1] * H * d + 4 * k_ptr[-1] * kv * d
            flops += 10 * pairs * H * d
        return {"bytes": nbytes, "flops": flops}
    own_len = _own_sizes(c)
    if c["op"] == "cache":
        rows = kv * sum(min(n, c["new"]) for n in own_len)
        padding = kv * c["batch"] * c["new"] - rows
        # rows in, codes and scales out; codes and scales in, rows out (rows
        # before a sequence's start: zeros)
        return {"bytes": 2 * (2 * rows * (2 * d + d + 1) + 2 * d * padding),
                "flops": 4 * rows * d}
    keys = sum(own_len) + c["prefix"]
    rows = c["batch"] * c["new"] * H
    pairs = sum(max(0, n - t) for n in own_len for t in range(c["new"]))
    pairs += c["prefix"] * c["batch"] * c["new"]
    return {"bytes": 2 * keys * kv * (d + 1) + rows * (4 * d + 4), "flops": 4 * pairs * H * d}


# ---- inputs -----------------------------------------------------------------------

def _exponents(x):
    """For each row (last dimension): the smallest e with max|x| <= 448 * 2^e."""
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0, torch.where(m <= 0.875, e - 9, e - 8), -127)
    return e.clamp(min=-127)


def _two_to(e):
    """2^e for whole e from -127 to 127, without rounding (a power function
    may be off by a unit in the last place, which moves values off a border)."""
    return ((e.to(torch.int32) + 128) << 23).clamp(max=254 << 23).view(torch.float32) \
        * torch.where(e < 127, 0.5, 1.0)


def _quantise(x):
    """Codes (8-bit floats) and biased exponents (bytes) of rows of x."""
    x = x.float()
    e = _exponents(x)
    return (x * _two_to(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _states(gen, shape):
    """Rows as a projection gives them: some channels much larger than others."""
    x = torch.randn(shape, generator=gen, device="cuda")
    return x * torch.exp(0.5 * torch.randn(shape[-1], generator=gen, device="cuda"))


def _tables(c, gen, n_pages_each, first):
    """A page table with the pages of every sequence in no order."""
    B = c["batch"]
    pages = first + torch.randperm(B * n_pages_each, generator=gen, device="cuda")
    return pages.to(torch.int32).view(B, n_pages_each)


def _inputs(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * int(seed) + 29)
    H, kv, d, dtype = c["heads"], c["kv"], c["d"], _TYPES[c["dtype"]]

    def rows(n, h):
        return torch.randn((n, h, d), generator=gen, device="cuda").to(dtype)

    if c["op"] == "cross":
        q, k, q_ptr, k_ptr = _cross_sizes(c)
        s = dict(q_len=q, k_len=k, q_ptr=q_ptr, k_ptr=k_ptr, Q=rows(q_ptr[-1], H),
                 K=rows(k_ptr[-1], kv), V=rows(k_ptr[-1], kv))
        if c.get("train"):
            s["dO"] = rows(q_ptr[-1], H)
        return s
    page, B, n = c["page"], c["batch"], c["new"]
    own_len = _own_sizes(c)
    each = -(-max(own_len) // page)
    shared = -(-c.get("prefix", 0) // page)
    n_pages = shared + B * each + 1
    s = dict(lens=torch.tensor(own_len, dtype=torch.int32, device="cuda"),
             table=_tables(c, gen, each, shared))
    if c["op"] == "cache":
        s["K"], s["V"] = (_states(gen, (B, n, kv, d)).to(dtype) for _ in "KV")
        for x in "kv":
            s[x] = torch.zeros((n_pages, kv, page, d), dtype=torch.uint8,
                               device="cuda").view(torch.float8_e4m3fn)
            s[x + "_exp"] = torch.zeros((n_pages, kv, page), dtype=torch.uint8, device="cuda")
        return s
    for x in "kv":
        s[x], s[x + "_exp"] = _quantise(_states(gen, (n_pages, kv, page, d)))
    s["Q"] = rows(B * n, H).view(B, n, H, d)
    s["prefix"] = (torch.arange(shared, dtype=torch.int32, device="cuda")
                   if shared else None)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2505_08098_amd as f3s
        if case["op"] == "cross":
            # the plan of the batch's lengths, which all layers share
            s["plan"] = f3s.CrossPlan(s["q_ptr"], s["k_ptr"], case["heads"], case["kv"],
                                      case["d"], q_len=s["q_len"], k_len=s["k_len"],
                                      device="cuda")
        else:
            s["cache"] = f3s.Cache(s["k"], s["v"], s["k_exp"], s["v_exp"])
    return s


# ---- one pass: the framework's calls -------------------------------------------------

def _run_own(s):
    import paper_2505_08098_amd as f3s
    c = s["case"]
    if c["op"] == "cross":
        O, lse = f3s.cross_forward(s["plan"], s["Q"], s["K"], s["V"])
        if not c.get("train"):
            return O, lse
        return (O, lse) + f3s.cross_backward(s["plan"], s["Q"], s["K"], s["V"], O, s["dO"],
                                             lse)
    if c["op"] == "cache":
        f3s.cache_write(s["cache"], s["K"], s["V"], s["table"], s["lens"])
        return f3s.cache_read(s["cache"], s["table"], s["lens"], c["new"], s["K"].dtype)
    return f3s.cache_attend(s["cache"], s["Q"], s["table"], s["lens"], prefix=s["prefix"],
                            prefix_len=c["prefix"])


# ---- one pass: plain torch in 32 bits ------------------------------------------------

def _pad(x, ptr, length, top):
    """Rows of every sequence, [B, heads, top, d] in 32 bits, zeros behind the
    last, and which are there [B, top]."""
    at = torch.arange(top, device="cuda")
    first = torch.tensor(ptr[:-1], device="cuda")[:, None]
    there = at < torch.tensor(length, device="cuda")[:, None]
    rows = torch.where(there, first + at, 0)
    return (x[rows].float() * there[..., None, None]).transpose(1, 2), rows, there


def _unpad(x, like, rows, there, dtype):
    """The rows that are there at their places, zeros at the others."""
    out = torch.zeros(like.shape[:x.dim() - 1], dtype=dtype, device="cuda")
    out[rows[there]] = x.transpose(1, 2)[there].to(dtype)
    return out


def _softmax(x, seen):
    """Probabilities and log-sum-exp of the scores that are seen, in place of
    x; rows without any: zeros and -inf."""
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    return p.div_(torch.where(total > 0, total, 1.0)), lse


def _cross(s):
    c = s["case"]
    H, kv, d = c["heads"], c["kv"], c["d"]
    g, B, dtype, scale = H // kv, c["batch"], _TYPES[c["dtype"]], 1.0 / math.sqrt(d)
    nq, nk = max(s["q_len"]), max(s["k_len"])
    K, k_rows, k_there = _pad(s["K"], s["k_ptr"], s["k_len"], nk)
    V = _pad(s["V"], s["k_ptr"], s["k_len"], nk)[0]
    Q, q_rows, q_there = _pad(s["Q"], s["q_ptr"], s["q_len"], nq)

    def grouped(x):  # the query heads of a key head one behind the other
        return x.reshape(B, kv, g * nq, d)

    def query_rows(x):
        return _unpad(x.reshape(B, H, nq, d), s["Q"], q_rows, q_there, dtype)

    Q = grouped(Q)
    P, lse = _softmax(torch.matmul(Q, K.transpose(-1, -2)).mul_(scale), k_there[:, None, None])
    O = torch.matmul(P, V)
    stats = torch.full(s["Q"].shape[:2], -math.inf, device="cuda")
    stats[q_rows[q_there]] = lse.view(B, H, nq).transpose(1, 2)[q_there]
    outs = (query_rows(O), stats)
    if not c.get("train"):
        return outs
    G = grouped(_pad(s["dO"], s["q_ptr"], s["q_len"], nq)[0])
    dV = torch.matmul(P.transpose(-1, -2), G)
    dS = torch.matmul(G, V.transpose(-1, -2))
    dS.sub_((G * O).sum(-1, keepdim=True)).mul_(P).mul_(scale)
    del P
    dQ = torch.matmul(dS, K)
    dK = torch.matmul(dS.transpose(-1, -2), Q)
    return outs + (query_rows(dQ),
                   _unpad(dK, s["K"], k_rows, k_there, dtype),
                   _unpad(dV, s["K"], k_rows, k_there, dtype))


def _slots(s, positions):
    """Page and place in it of positions [B, n] of every sequence."""
    page = s["case"]["page"]
    return torch.gather(s["table"].long(), 1, positions // page), positions % page


def _values(s, x, pages, places):
    """Cached rows [..., heads, d] in 32 bits."""
    codes = s[x].view(torch.uint8)[pages, :, places].view(torch.float8_e4m3fn).float()
    e = s[x + "_exp"][pages, :, places].to(torch.int32) - 127
    return codes * _two_to(e)[..., None]


def _cache(s):
    c = s["case"]
    n = c["new"]
    at = s["lens"].long()[:, None] - n + torch.arange(n, device="cuda")
    there = at >= 0
    pages, places = _slots(s, at.clamp(min=0))
    out = []
    for x, rows in (("k", s["K"]), ("v", s["V"])):
        codes, e = _quantise(rows)
        s[x].view(torch.uint8)[pages[there], :, places[there]] = \
            codes.view(torch.uint8)[there]
        s[x + "_exp"][pages[there], :, places[there]] = e[there]
        back = _values(s, x, pages, places)
        out.append(back.masked_fill_(~there[..., None, None], 0.0).to(rows.dtype))
    return tuple(out)


def _attend(s):
    c = s["case"]
    H, kv, d, B, n = c["heads"], c["kv"], c["d"], c["batch"], c["new"]
    g, scale, P = H // kv, 1.0 / math.sqrt(d), c["prefix"]
    lens = s["lens"].long()
    at = torch.arange(s["table"].shape[1] * c["page"], device="cuda")
    pages, places = _slots(s, at.expand(B, -1))
    # query rows [B, kv, g * n, d]: the heads of a group, then the tokens
    Q = s["Q"].float().transpose(1, 2).reshape(B, kv, g * n, d)
    x = torch.matmul(Q, _values(s, "k", pages, places).permute(0, 2, 3, 1)).mul_(scale)
    last = lens[:, None] - n + torch.arange(n, device="cuda")
    seen = (at <= last[..., None])[:, None, None].expand(B, kv, g, n, -1).flatten(2, 3)
    if P:
        spot = torch.arange(P, device="cuda")
        shared = s["prefix"].long()[spot // c["page"]], spot % c["page"]
        first = torch.matmul(Q.transpose(0, 1).reshape(kv, -1, d),
                             _values(s, "k", *shared).permute(1, 2, 0)).mul_(scale)
        x = torch.cat([first.view(kv, B, g * n, P).transpose(0, 1), x], -1)
        seen = torch.cat([seen.new_ones(()).expand(B, kv, g * n, P), seen], -1)
    p, lse = _softmax(x, seen)
    O = torch.matmul(p[..., P:], _values(s, "v", pages, places).transpose(1, 2))
    if P:
        front = p[..., :P].transpose(0, 1).reshape(kv, -1, P)
        O += torch.matmul(front, _values(s, "v", *shared).transpose(0, 1)) \
            .view(kv, B, g * n, d).transpose(0, 1)
    return (O.reshape(B, H, n, d).transpose(1, 2).to(s["Q"].dtype),
            lse.reshape(B, H, n).transpose(1, 2).contiguous())


def run(state):
    if own:
        return _run_own(state)
    return {"cross": _cross, "cache": _cache, "attend": _attend}[state["case"]["op"]](state)


# ---- the same in 64 bits, one sequence after the other ---------------------------------

def _exact_rows(Q, K, V, seen=None):
    """softmax(Q K^T / sqrt(d)) V of one head in 64 bits: O, lse, P."""
    x = Q @ K.T / math.sqrt(Q.shape[1])
    if seen is not None:
        x = torch.where(seen, x, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    return p @ V, lse, p


def _exact_cross(c, s):
    H, d = c["heads"], c["d"]
    g = H // c["kv"]
    Q, K, V = (s[x].double() for x in "QKV")
    O, dQ, dK, dV = (torch.zeros_like(x) for x in (Q, Q, K, V))
    lse = torch.full(Q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        i = slice(s["q_ptr"][b], s["q_ptr"][b] + s["q_len"][b])
        j = slice(s["k_ptr"][b], s["k_ptr"][b] + s["k_len"][b])
        for h in range(H):
            k, v = K[j, h // g], V[j, h // g]
            O[i, h], lse[i, h], p = _exact_rows(Q[i, h], k, v)
            if c.get("train"):
                G = s["dO"][i, h].double()
                dS = p * (G @ v.T - (G * O[i, h]).sum(1, keepdim=True)) / math.sqrt(d)
                dQ[i, h] = dS @ k
                dK[j, h // g] += dS.T @ Q[i, h]
                dV[j, h // g] += p.T @ G
    return (O, lse, dQ, dK, dV) if c.get("train") else (O, lse)


def _code_values():
    """The 256 values of an 8-bit float with 4 exponent and 3 fraction bits."""
    b = torch.arange(256, dtype=torch.float64, device="cuda")
    sign, e, f = 1 - 2 * (b // 128), b % 128 // 8, b % 8
    v = torch.where(e > 0, (1 + f / 8) * 2.0 ** (e - 7), f / 8 * 2.0 ** -6)
    return sign * torch.where(b % 128 == 127, math.nan, v)


def _power(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_round(x):
    """Rows of x, each rounded to the nearest value that a code and the row's
    power of two give, to the even code in the middle."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448)).clamp(min=-127)
    # (log2 may be off by one unit next to a whole number)
    e = torch.where(448 * _power(e - 1) >= top, e - 1, e)
    e = torch.where(448 * _power(e) < top, e + 1, e).clamp(min=-127)
    y = x * _power(-e)
    octave = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    octave = torch.where(_power(octave) > y.abs(), octave - 1, octave)
    octave = torch.where(_power(octave + 1) <= y.abs(), octave + 1, octave).clamp(min=-6)
    return torch.round(y * _power(3 - octave)) * _power(octave - 3) * _power(e)


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["op"] == "cross":
        return _exact_cross(c, s)
    H, kv, d, page, n = c["heads"], c["kv"], c["d"], c["page"], c["new"]
    lens = s["lens"].tolist()
    if c["op"] == "cache":
        out = [_exact_round(s[x]) for x in "KV"]
        for b, m in enumerate(lens):
            for x in out:
                x[b, :max(0, n - m)] = 0
        return tuple(out)
    value = _code_values()

    def rows(x, pages, m):
        """Cached rows [m, kv, d] of a list of pages."""
        codes = value[s[x].view(torch.uint8)[pages.long()].long()]
        e = s[x + "_exp"][pages.long()].double() - 127
        return (codes * _power(e)[..., None]).transpose(1, 2).reshape(-1, kv, d)[:m]

    front = [rows(x, s["prefix"], c["prefix"]) for x in "kv"] if c["prefix"] else None
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["Q"].shape[:-1], dtype=torch.float64, device="cuda")
    for b, m in enumerate(lens):
        k, v = (rows(x, s["table"][b], m) for x in "kv")
        if front:
            k, v = torch.cat([front[0], k]), torch.cat([front[1], v])
        # token t sees the prefix and the first m - n + 1 + t own keys
        limit = c["prefix"] + m - n + 1 + torch.arange(n, device="cuda")
        seen = torch.arange(len(k), device="cuda") < limit[:, None]
        for h in range(H):
            O[b, :, h], lse[b, :, h], _ = _exact_rows(s["Q"][b, :, h].double(),
                                                      k[:, h * kv // H], v[:, h * kv // H],
                                                      seen)
    return O, lse
