"""Attention of generated tokens to what they may see, and the cache's bookkeeping,
as programs use them.

Five operators:

window   causal self-attention of a ragged batch in which a token sees the newest
         `window` tokens and the first `sinks` ones, with its gradients
recent   the same for the newest tokens of a batch over the 8-bit paged cache
tree     the tokens of a drafted tree attend to the cache, to a prefix that the
         batch shares and to their own ancestors in the tree
keep     the accepted tokens of a draft move to the front of it in the cache
pages    pages of the cache given to sequences that grow and taken from those that
         shrink, with the places of the newest tokens

``own`` false: the operators in plain torch, in 32 bits.  ``own`` true: the
framework's calls.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _case(name, op, **sizes):
    """len, own, new_own: the shortest and the longest of the batch's lengths."""
    c = dict(op=op)
    if op != "pages":
        c.update(heads=8, kv=8, d=64, dtype="f16")
    for key, v in sizes.items():
        if key in ("len", "own"):
            c[key + "_least"], c[key] = v
        else:
            c[key] = v
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a training step on a small batch of sentences: latency
        _case("window_small", "window", batch=8, len=(20, 130), window=64, sinks=0, train=True),
        # a training step on padded documents that fit the window: causal attention
        _case("window_causal_padded", "window", heads=12, kv=12, batch=16, len=(300, 1025),
              window=2048, sinks=0, train=True, padded=True),
        # a very long document read at once, shared key heads: the matrix units count
        _case("window_long", "window", heads=32, kv=8, d=128, dtype="bf16", batch=1,
              len=(32749, 32749), window=4096, sinks=4),
        # training on long documents, ragged, four query heads to a key head
        _case("window_long_train", "window", heads=16, kv=4, d=128, dtype="bf16", batch=2,
              len=(8001, 8190), window=1024, sinks=16, train=True),
        # one token for each sequence of a ragged batch: bytes of the window
        _case("recent_token", "recent", heads=32, kv=8, d=128, dtype="bf16", batch=64, new=1,
              page=64, own=(500, 20000), window=4096, sinks=4),
        # a part of two long prompts: the matrix units count
        _case("recent_prompt", "recent", heads=16, kv=4, d=128, batch=2, new=2000, page=64,
              own=(5000, 9000), window=4000, sinks=4),
        # a small tree behind one sequence of ordinary length: latency
        _case("tree_one", "tree", batch=1, new=8, page=16, own=(4001, 4001), prefix=0),
        # large trees for a ragged batch behind a prompt that it shares
        _case("tree_batch", "tree", heads=32, kv=8, d=128, dtype="bf16", batch=16, new=63,
              page=64, own=(500, 8192), prefix=2001),
        # what one sequence accepts of a small draft: latency
        _case("keep_one", "keep", batch=1, new=8, page=16, own=(4001, 4001), most=5),
        # a large batch's accepted tokens of large trees
        _case("keep_batch", "keep", kv=8, d=128, dtype="bf16", batch=256, new=64, page=64,
              own=(100, 3000), most=9),
        # a draft's tokens get their places, those that need it a page, and give it back
        _case("pages_step", "pages", batch=256, page=64, own=(100, 8000), new=5, turn=0.0,
              spare=1.0),
        # much of a large batch ends and other requests begin; pages are short
        _case("pages_turn", "pages", batch=4096, page=16, own=(200, 8000), new=256, turn=0.5,
              spare=0.2),
    ]


# what the listed cases need at most: operations, bytes, values of the plain forms'
# scores, and entries of a table or of its newest tokens' places
_MOST_FLOPS = 4 * 126_000_000 * 32 * 128
_MOST_BYTES = 700 << 20
_MOST_SCORES = 32749 * 4355 * 32
_MOST_ENTRIES = 4096 * 512


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("window", "window", "recent", "tree", "keep", "pages"))
        if op == "pages":
            top = _log_int(rng, 20, 32768)
            c = _case(None, op, batch=_log_int(rng, 1, 4096), page=rng.choice((16, 32, 64, 128, 256)),
                      own=(top // 20, top), new=_log_int(rng, 1, 256),
                      turn=rng.choice((0.0, 0.0, 0.1, 0.5)), spare=rng.choice((0.2, 1.0)))
            entries = c["batch"] * max(_max_pages(c), c["new"])
            if entries <= _MOST_ENTRIES and work(c)["bytes"] <= _MOST_BYTES:
                return c
            continue
        kv = rng.choice((1, 2, 3, 4, 8))
        sizes = dict(kv=kv, heads=kv * rng.choice((1, 1, 2, 4, 5, 8)),
                     d=rng.choice((32, 64, 64, 96, 128, 128, 256)),
                     dtype=rng.choice(("f16", "bf16")))
        if op in ("window", "recent"):
            sizes.update(window=_log_int(rng, 16, 8192),
                         sinks=rng.choice((0, 0, 1, 4, 4, 16, 100)))
        if op == "window":
            n = _log_int(rng, 20, 32768)
            sizes.update(batch=_log_int(rng, 1, 64), len=((n + 2) // 3, n))
            if rng.random() < 0.6:
                sizes["train"] = True
            if rng.random() < 0.3:
                sizes["padded"] = True
            if rng.random() < 0.2:
                # the newest tokens only
                sizes["new"] = _log_int(rng, 1, n)
        else:
            top = _log_int(rng, 20, 65536)
            sizes.update(batch=_log_int(rng, 1, 128), page=rng.choice((16, 32, 64, 128, 256)),
                         own=(top // 8, top))
            if op == "recent":
                sizes["new"] = 1 if rng.random() < 0.5 else _log_int(rng, 2, 4096)
            else:
                sizes["new"] = _log_int(rng, 2, 160)
                if op == "tree":
                    sizes["prefix"] = rng.choice((0, 1)) * _log_int(rng, 20, 16384)
                else:
                    sizes["heads"] = kv
                    sizes["most"] = rng.randint(1, min(16, sizes["new"]))
        c = _case(None, op, **sizes)
        w = work(c)
        if (w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES
                and _scores(c) <= _MOST_SCORES):
            return c


# ---- sizes ------------------------------------------------------------------------

def _lengths(lo, hi, n, turn=0):
    """n lengths from lo to hi, both among them where n > 1, in mixed order."""
    if n == 1:
        return [hi]
    step = next(s for s in (37, 41, 43, 47) if math.gcd(s, n) == 1)
    return [lo + (hi - lo) * ((i * step + turn) % n) // (n - 1) for i in range(n)]


def _sums(x):
    return [0] + np.cumsum(x).tolist()


def _window_sizes(c):
    """Query and key rows of every sequence, and the first row of each in Q and in K
    and V: one behind the other, or padded to the longest."""
    k = _lengths(c["len_least"], c["len"], c["batch"])
    q = [min(x, c.get("new", x)) for x in k]
    if c.get("padded"):
        return q, k, [max(q) * i for i in range(c["batch"] + 1)], \
            [max(k) * i for i in range(c["batch"] + 1)]
    return q, k, _sums(q), _sums(k)


def _own_sizes(c):
    return _lengths(c["own_least"], c["own"], c["batch"])


_BLOCK = 256  # query tokens of a block of the plain form


def _scores(c):
    """Scores that the plain form keeps."""
    if c["op"] == "window":
        q, k = _window_sizes(c)[:2]
        block = min(_BLOCK, max(q))
        rows = c["batch"] * -(-max(q) // block) * block
        return rows * c["heads"] * (min(c["window"], max(k)) + block + min(c["sinks"], max(k)))
    rows = c["batch"] * c["new"] * c["heads"]
    if c["op"] == "recent":
        return rows * (min(c["window"], c["own"]) + c["new"] + c["sinks"])
    return rows * (c["own"] + c.get("prefix", 0))


def _seen_keys(first, last, window, sinks):
    """Keys that the tokens at positions first .. last see, one after the other."""
    p = np.arange(max(first, 0), last + 1, dtype=np.int64)
    return np.minimum(p + 1, window) + np.minimum(sinks, np.maximum(0, p + 1 - window))


def _read_keys(first, last, window, sinks):
    """Keys that any of them sees."""
    if last < 0:
        return 0
    least = max(0, max(first, 0) - window + 1)
    return last + 1 - least + min(sinks, least) if window else min(sinks, last + 1)


def _max_pages(c):
    """Pages of a row of the table: for the longest and its newest tokens."""
    return -(-(c["own"] + c["new"]) // c["page"])


def _page_lens(c):
    """Lengths before and after: every sequence takes `new` tokens more, but every
    few of them (the share `turn`) end, and as many that are empty begin."""
    now = _own_sizes(c)
    then = [n + c["new"] for n in now]
    if c["turn"]:
        every = round(1 / c["turn"])
        for i in range(0, len(now), 2 * every):
            then[i] = 0
        for i in range(every, len(now), 2 * every):
            now[i] = 0
    return now, then


def work(case):
    c = case
    if c["op"] == "pages":
        now, then = _page_lens(c)
        moved = sum(abs(-(-b // c["page"]) - -(-a // c["page"])) for a, b in zip(now, then))
        # lengths in, pages from one list to the other, lengths and places out; and back
        return {"bytes": 2 * (12 * c["batch"] + 8 * moved) + 8 * c["batch"] * c["new"],
                "flops": 0}
    H, kv, d = c["heads"], c["kv"], c["d"]
    if c["op"] == "window":
        q, k, q_ptr, k_ptr = _window_sizes(c)
        pairs = sum(int(_seen_keys(b - a, b - 1, c["window"], c["sinks"]).sum())
                    for a, b in zip(q, k))
        keys = sum(_read_keys(b - a, b - 1, c["window"], c["sinks"]) for a, b in zip(q, k))
        # Q, K, V in, O and the log-sum-exp out
        nbytes = 2 * sum(q) * H * d + 4 * keys * kv * d + q_ptr[-1] * H * (2 * d + 4)
        flops = 4 * pairs * H * d
        if c.get("train"):
            # dO in, dQ, dK and dV out
            nbytes += 2 * sum(q) * H * d + 2 * q_ptr[-1] * H * d + 4 * k_ptr[-1] * kv * d
            flops += 10 * pairs * H * d
        return {"bytes": nbytes, "flops": flops}
    lens, n = _own_sizes(c), c["new"]
    if c["op"] == "keep":
        rows = c["batch"] * c["new"] * kv
        kept = c["batch"] * c["most"] * kv
        # rows in, codes and powers out; kept ones moved; read back
        return {"bytes": 2 * (rows * (2 * d + d + 1) + 2 * kept * (d + 1)
                              + kept * (d + 1 + 2 * d)), "flops": 0}
    rows = c["batch"] * n * H
    if c["op"] == "recent":
        pairs = sum(int(_seen_keys(m - n, m - 1, c["window"], c["sinks"]).sum()) for m in lens)
        keys = sum(_read_keys(m - n, m - 1, c["window"], c["sinks"]) for m in lens)
    else:
        # of a tree's tokens a token sees about as many as the tree is deep
        depth = max(1, int(2 * math.sqrt(n)))
        pairs = sum((max(0, m - n) + depth) * n for m in lens) + c["prefix"] * c["batch"] * n
        keys = sum(lens) + c["prefix"]
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


def _tables(batch, gen, n_pages_each, first):
    """A page table with the pages of every sequence in no order."""
    pages = first + torch.randperm(batch * n_pages_each, generator=gen, device="cuda")
    return pages.to(torch.int32).view(batch, n_pages_each)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pages_inputs(c, gen):
    now, then = _page_lens(c)
    B, M = c["batch"], _max_pages(c)
    held = -(-_ints(now).long() // c["page"])
    extra = sum(max(0, -(-b // c["page"]) - -(-a // c["page"])) for a, b in zip(now, then))
    n_pages = sum(-(-a // c["page"]) for a in now) + max(1, int(extra * c["spare"]))
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    there = torch.arange(M, device="cuda") < held[:, None]
    rank = torch.cumsum(there.flatten(), 0).view(B, M) - 1
    table = torch.where(there, order[rank.clamp(min=0)], -1)
    used = int(held.sum())
    # the free pages stand at the front of their list
    free = torch.cat([order[used:], order.new_full((used,), -1)])
    return dict(lens=_ints(now), then=_ints(then), table=table.contiguous(), free=free,
                count=_ints([n_pages - used]))


def _inputs(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * int(seed) + 31)
    if c["op"] == "pages":
        return _pages_inputs(c, gen)
    H, kv, d, dtype = c["heads"], c["kv"], c["d"], _TYPES[c["dtype"]]

    def rows(n, h):
        return torch.randn((n, h, d), generator=gen, device="cuda").to(dtype)

    if c["op"] == "window":
        q, k, q_ptr, k_ptr = _window_sizes(c)
        s = dict(q_len=q, k_len=k, q_ptr=q_ptr, k_ptr=k_ptr, Q=rows(q_ptr[-1], H),
                 K=rows(k_ptr[-1], kv), V=rows(k_ptr[-1], kv))
        if c.get("train"):
            s["dO"] = rows(q_ptr[-1], H)
        return s
    page, B, n = c["page"], c["batch"], c["new"]
    lens = _own_sizes(c)
    if c["op"] == "keep":  # (the draft's tokens are all there)
        lens = [max(m, n) for m in lens]
    each = -(-max(lens) // page)
    shared = -(-c.get("prefix", 0) // page)
    n_pages = shared + B * each + 1
    s = dict(lens=_ints(lens), table=_tables(B, gen, each, shared))
    for x in "kv":
        s[x], s[x + "_exp"] = _quantise(_states(gen, (n_pages, kv, page, d)))
    if c["op"] == "keep":
        s["K"], s["V"] = (_states(gen, (B, n, kv, d)).to(dtype) for _ in "KV")
        # some of the draft's tokens, in order; behind them -1
        picks = torch.rand((B, n), generator=gen, device="cuda").topk(c["most"]).indices
        picks = picks.sort().values
        kept = torch.randint(0, c["most"] + 1, (B, 1), generator=gen, device="cuda")
        s["picks"] = torch.where(torch.arange(c["most"], device="cuda") < kept, picks,
                                 -1).to(torch.int32).contiguous()
        return s
    s["Q"] = rows(B * n, H).view(B, n, H, d)
    if c["op"] == "tree":
        s["prefix"] = (torch.arange(shared, dtype=torch.int32, device="cuda")
                       if shared else None)
        # every token's parent is one of those before it, or none (-1): a draft
        # several tokens wide and deep
        at = torch.arange(n, device="cuda").expand(B, n)
        back = torch.randint(1, max(2, int(2 * math.sqrt(n)) + 1), (B, n), generator=gen,
                             device="cuda")
        s["parents"] = (at - back).clamp(min=-1).to(torch.int32).contiguous()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2505_08098_amd as f3s
        c = case
        if c["op"] == "window":
            # the plan of the batch's lengths, which all layers share
            s["plan"] = f3s.WindowPlan(s["q_ptr"], s["k_ptr"], c["heads"], c["kv"], c["d"],
                                       window=c["window"], sinks=c["sinks"], q_len=s["q_len"],
                                       k_len=s["k_len"], device="cuda")
        elif c["op"] == "pages":
            s["pool"] = f3s.PagePool(s["free"], s["count"], c["page"])
        else:
            s["cache"] = f3s.Cache(s["k"], s["v"], s["k_exp"], s["v_exp"])
    return s


# ---- one pass: the framework's calls -------------------------------------------------

def _run_own(s):
    import paper_2505_08098_amd as f3s
    c = s["case"]
    if c["op"] == "window":
        O, lse = f3s.window_forward(s["plan"], s["Q"], s["K"], s["V"])
        if not c.get("train"):
            return O, lse
        return (O, lse) + f3s.window_backward(s["plan"], s["Q"], s["K"], s["V"], O, s["dO"],
                                              lse)
    if c["op"] == "recent":
        return f3s.cache_attend_window(s["cache"], s["Q"], s["table"], s["lens"],
                                       window=c["window"], sinks=c["sinks"])
    if c["op"] == "tree":
        return f3s.cache_attend_tree(s["cache"], s["Q"], s["table"], s["lens"], s["parents"],
                                     prefix=s["prefix"], prefix_len=c["prefix"])
    if c["op"] == "keep":
        # the draft enters the cache; what is accepted of it stays; the next layer's form
        f3s.cache_write(s["cache"], s["K"], s["V"], s["table"], s["lens"])
        lens = f3s.cache_keep(s["cache"], s["table"], s["lens"], c["new"], s["picks"])
        return (lens,) + f3s.cache_read(s["cache"], s["table"], lens, c["most"], s["K"].dtype)
    # pages for what comes, and back from those that are given up
    got, slots = f3s.pages_assign(s["pool"], s["table"], s["lens"], s["then"], n=c["new"])
    back, _ = f3s.pages_assign(s["pool"], s["table"], got, s["lens"])
    return got, slots, back, s["table"], s["pool"].free, s["pool"].count


# ---- one pass: plain torch in 32 bits ------------------------------------------------

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


def _window(s):
    c = s["case"]
    H, kv, d, B = c["heads"], c["kv"], c["d"], c["batch"]
    g, dtype, scale = H // kv, _TYPES[c["dtype"]], 1.0 / math.sqrt(d)
    q_len, k_len = (torch.tensor(s[x], device="cuda") for x in ("q_len", "k_len"))
    q_ptr, k_ptr = (torch.tensor(s[x][:-1], device="cuda") for x in ("q_ptr", "k_ptr"))
    block = min(_BLOCK, max(s["q_len"]))
    n = -(-max(s["q_len"]) // block)
    # tokens [B, n, block] and their positions
    i = torch.arange(n * block, device="cuda").view(n, block).expand(B, n, block)
    there = i < q_len[:, None, None]
    p = i + (k_len - q_len)[:, None, None]
    rows = torch.where(there, q_ptr[:, None, None] + i, 0)
    # keys that a block's tokens may see [B, n, m]: the sinks, then the window's
    width = min(c["window"], max(s["k_len"]))
    few = min(c["sinks"], max(s["k_len"]))
    near = p[..., :1] - width + 1 + torch.arange(width + block - 1, device="cuda")
    far = torch.arange(few, device="cuda").expand(B, n, few)
    j = torch.cat([far, near], -1)
    real = torch.cat([far >= 0, near >= few], -1)
    seen = (real[:, :, None] & (j[:, :, None] <= p[..., None])
            & ((j[:, :, None] > p[..., None] - c["window"]) | (j[:, :, None] < c["sinks"])))
    seen = seen[:, :, None, None].expand(B, n, kv, g, block, -1).flatten(3, 4)
    k_rows = k_ptr[:, None, None] + torch.minimum(j, k_len[:, None, None] - 1).clamp(min=0)

    def queries(x):  # the query heads of a key head one behind the other
        x = x[rows].float() * there[..., None, None]
        return x.view(B, n, block, kv, g, d).permute(0, 1, 3, 4, 2, 5).reshape(
            B, n, kv, g * block, d)

    def out(x, value):  # rows that are there at their places
        y = torch.full((s["Q"].shape[0], H) + x.shape[5:], value, device="cuda",
                       dtype=dtype if x.dim() > 5 else torch.float32)
        y[rows[there]] = x.movedim(4, 2).reshape((B, n, block, H) + x.shape[5:])[there].to(
            y.dtype)
        return y

    K, V = (s[x][k_rows].float().transpose(2, 3) for x in "KV")
    Q = queries(s["Q"])
    P, lse = _softmax(torch.matmul(Q, K.transpose(-1, -2)).mul_(scale), seen)
    O = torch.matmul(P, V)
    outs = (out(O.view(B, n, kv, g, block, d), 0.0),
            out(lse.view(B, n, kv, g, block), -math.inf))
    if not c.get("train"):
        return outs
    G = queries(s["dO"])
    dV = torch.matmul(P.transpose(-1, -2), G)
    dS = torch.matmul(G, V.transpose(-1, -2))
    dS.sub_((G * O).sum(-1, keepdim=True)).mul_(P).mul_(scale)
    del P
    dQ = torch.matmul(dS, K)
    dK = torch.matmul(dS.transpose(-1, -2), Q)

    def keys(x):  # summed over the blocks that see a key
        y = torch.zeros(s["K"].shape, dtype=torch.float32, device="cuda")
        y.index_add_(0, k_rows.flatten(), x.transpose(2, 3).reshape(-1, kv, d))
        return y.to(dtype)

    return outs + (out(dQ.view(B, n, kv, g, block, d), 0.0), keys(dK), keys(dV))


def _slots(s, positions):
    """Page and place in it of positions [B, n] of every sequence."""
    page = s["case"]["page"]
    return torch.gather(s["table"].long(), 1, positions // page), positions % page


def _values(s, x, pages, places):
    """Cached rows [..., heads, d] in 32 bits."""
    codes = s[x].view(torch.uint8)[pages, :, places].view(torch.float8_e4m3fn).float()
    e = s[x + "_exp"][pages, :, places].to(torch.int32) - 127
    return codes * _two_to(e)[..., None]


def _cached(s, at, seen):
    """The newest tokens' attention to the keys at positions at [B, m] of their own and to
    the prefix; seen [B, n, m]."""
    c = s["case"]
    H, kv, d, B, n = c["heads"], c["kv"], c["d"], c["batch"], c["new"]
    g, scale, P = H // kv, 1.0 / math.sqrt(d), c.get("prefix", 0)
    pages, places = _slots(s, at)
    # query rows [B, kv, g * n, d]: the heads of a group, then the tokens
    Q = s["Q"].float().transpose(1, 2).reshape(B, kv, g * n, d)
    x = torch.matmul(Q, _values(s, "k", pages, places).permute(0, 2, 3, 1)).mul_(scale)
    seen = seen[:, None, None].expand(B, kv, g, n, -1).flatten(2, 3)
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


def _recent(s):
    c = s["case"]
    B, n, cap = c["batch"], c["new"], s["table"].shape[1] * c["page"]
    width, few = min(c["window"], cap), min(c["sinks"], cap)
    last = s["lens"].long()[:, None] - n + torch.arange(n, device="cuda")
    near = last[:, :1] - width + 1 + torch.arange(width + n - 1, device="cuda")
    at = torch.cat([torch.arange(few, device="cuda").expand(B, few), near], 1)
    seen = torch.cat([near.new_ones((B, few)), near >= few], 1)[:, None].bool() \
        & (at[:, None] <= last[..., None]) \
        & ((at[:, None] > last[..., None] - c["window"]) | (at[:, None] < c["sinks"]))
    return _cached(s, at.clamp(0, cap - 1), seen)


def _ancestors(parents):
    """[B, n, n]: whether token j is token i or an ancestor of it."""
    n = parents.shape[1]
    at = torch.arange(n, device="cuda")
    reach = ((at == at[:, None]) | (at == parents.long()[..., None])).float()
    for _ in range(max(1, n.bit_length())):  # twice as far each time
        reach = (torch.matmul(reach, reach) > 0).float()
    return reach > 0


def _tree(s):
    c = s["case"]
    n = c["new"]
    at = torch.arange(s["table"].shape[1] * c["page"], device="cuda").expand(c["batch"], -1)
    first = s["lens"].long()[:, None] - n            # of the draft
    node = (at - first).clamp(0, n - 1)
    inside = torch.gather(_ancestors(s["parents"]), 2, node[:, None].expand(-1, n, -1))
    own_keys = (at < s["lens"][:, None])[:, None]
    # (a token with a position before the sequence's start is padding)
    there = (first + torch.arange(n, device="cuda") >= 0)[..., None]
    return _cached(s, at, own_keys & there & torch.where((at < first)[:, None], True, inside))


def _keep(s):
    c = s["case"]
    n, m = c["new"], c["most"]
    first = s["lens"].long()[:, None] - n
    to = _slots(s, first + torch.arange(n, device="cuda"))
    kept = (s["picks"] >= 0).sum(1, dtype=torch.int32)
    lens = s["lens"] - n + kept
    # the token that stands at each of the first places of the draft then
    moves = torch.arange(m, device="cuda") < kept[:, None]
    take = torch.where(moves, s["picks"].long(), torch.arange(m, device="cuda"))
    at = lens.long()[:, None] - m + torch.arange(m, device="cuda")
    read = _slots(s, at.clamp(min=0))
    out = [lens]
    for x, rows in (("k", s["K"]), ("v", s["V"])):
        codes, e = _quantise(rows)
        s[x].view(torch.uint8)[to[0], :, to[1]] = codes.view(torch.uint8)
        s[x + "_exp"][to[0], :, to[1]] = e
        from_ = _slots(s, first + take)
        codes, e = s[x].view(torch.uint8)[from_[0], :, from_[1]], s[x + "_exp"][from_[0], :,
                                                                                from_[1]]
        s[x].view(torch.uint8)[to[0][:, :m], :, to[1][:, :m]] = codes
        s[x + "_exp"][to[0][:, :m], :, to[1][:, :m]] = e
        back = _values(s, x, *read)
        out.append(back.masked_fill_((at < 0)[..., None, None], 0.0).to(rows.dtype))
    return tuple(out)


def _assign(s, old, new, n):
    """Pages for lengths `new` where those of `old` are held: what is released goes onto the
    list's end, what is needed comes from there, both in the order of sequences."""
    page, table, free, count = s["case"]["page"], s["table"], s["free"], s["count"]
    B, M = table.shape
    old, new = (x.long().clamp(0, M * page) for x in (old, new))
    have, want = -(-old // page), -(-new // page)
    e = torch.arange(M, device="cuda")
    over = (e >= want[:, None]) & (e < have[:, None])
    gone = over & (table >= 0) & (table < free.numel())
    room = torch.cat([free, free.new_zeros(1)])
    place = torch.where(gone.flatten(), count.long() + torch.cumsum(gone.flatten(), 0) - 1,
                        free.numel())
    room[place] = table.flatten()
    listed_ = count.long() + gone.sum()
    need = (e >= have[:, None]) & (e < want[:, None])
    rank = torch.cumsum(need.flatten(), 0).view(B, M) - 1
    given = torch.minimum(need.sum(), listed_)
    served = need & (rank < given)
    pages = room[(listed_ - given + rank).clamp(0, free.numel() - 1)]
    table.copy_(torch.where(over, -1, torch.where(need, torch.where(served, pages, -1), table)))
    free.copy_(room[:-1])
    count.copy_(listed_ - given)
    got = torch.minimum(new, (torch.minimum(have, want) + served.sum(1)) * page)
    at = new[:, None] - n + torch.arange(n, device="cuda")
    there = (at >= 0) & (at < got[:, None])
    its = torch.gather(table, 1, torch.where(there, at // page, 0)).long()
    slots = torch.where(there & (its >= 0) & (its < free.numel()), its * page + at % page, -1)
    return got.to(torch.int32), slots


def _pages(s):
    got, slots = _assign(s, s["lens"], s["then"], s["case"]["new"])
    back, _ = _assign(s, got, s["lens"], 0)
    return got, slots, back, s["table"], s["free"], s["count"]


def run(state):
    if own:
        return _run_own(state)
    return {"window": _window, "recent": _recent, "tree": _tree, "keep": _keep,
            "pages": _pages}[state["case"]["op"]](state)


# ---- the same in 64 bits, one sequence after the other ---------------------------------

def _exact_rows(Q, K, V, seen):
    """softmax(Q K^T / sqrt(d)) V of one head in 64 bits over what is seen: O, lse, P."""
    x = torch.where(seen, Q @ K.T / math.sqrt(Q.shape[1]), -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    return p @ V, lse, p


def _exact_window(c, s):
    H, d, W, S = c["heads"], c["d"], c["window"], c["sinks"]
    g = H // c["kv"]
    Q, K, V = (s[x].double() for x in "QKV")
    O, dQ, dK, dV = (torch.zeros_like(x) for x in (Q, Q, K, V))
    lse = torch.full(Q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        nq, nk = s["q_len"][b], s["k_len"][b]
        for t in range(0, nq, 2048):
            p = torch.arange(nk - nq + t, nk - nq + min(nq, t + 2048), device="cuda")[:, None]
            # keys from the first that the rows' windows hold, with the sinks before it
            near = max(0, nk - nq + t - W + 1)
            j = torch.cat([torch.arange(min(S, near), device="cuda"),
                           torch.arange(near, nk - nq + min(nq, t + 2048), device="cuda")])
            seen = (j <= p) & ((j < S) | (p - j < W))
            i = slice(s["q_ptr"][b] + t, s["q_ptr"][b] + min(nq, t + 2048))
            j = j + s["k_ptr"][b]
            for h in range(H):
                k, v = K[j, h // g], V[j, h // g]
                O[i, h], lse[i, h], P = _exact_rows(Q[i, h], k, v, seen)
                if c.get("train"):
                    G = s["dO"][i, h].double()
                    dS = P * (G @ v.T - (G * O[i, h]).sum(1, keepdim=True)) / math.sqrt(d)
                    dQ[i, h] = dS @ k
                    dK[j, h // g] += dS.T @ Q[i, h]
                    dV[j, h // g] += P.T @ G
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


def _exact_keep(c, s, rows):
    n, m = c["new"], c["most"]
    draft = [_exact_round(s[x]) for x in "KV"]
    out = [torch.zeros((c["batch"], m) + x.shape[2:], dtype=torch.float64, device="cuda")
           for x in draft]
    for b, (length, picks) in enumerate(zip(s["lens"].tolist(), s["picks"].tolist())):
        kept = [p for p in picks if p >= 0]
        for x, new, to in zip("kv", draft, out):
            before = max(0, min(m - len(kept), length - n))  # tokens ahead of the draft
            if before:
                to[b, m - len(kept) - before: m - len(kept)] = \
                    rows(x, s["table"][b], length - n)[-before:]
            to[b, m - len(kept):] = new[b, kept]
    return (None,) + tuple(out)


def exact(case, seed):
    c = case
    if c["op"] == "pages":
        return None
    s = _inputs(case, seed)
    if c["op"] == "window":
        return _exact_window(c, s)
    H, kv, d, n = c["heads"], c["kv"], c["d"], c["new"]
    if c["op"] != "keep" and c["batch"] * H * (c["own"] + c.get("prefix", 0)) * n > 1 << 33:
        return None
    value = _code_values()

    def rows(x, pages, m):
        """Cached rows [m, kv, d] of a list of pages."""
        pages = pages[: -(-m // c["page"])].long()
        codes = value[s[x].view(torch.uint8)[pages].long()]
        e = s[x + "_exp"][pages].double() - 127
        return (codes * _power(e)[..., None]).transpose(1, 2).reshape(-1, kv, d)[:m]

    if c["op"] == "keep":
        return _exact_keep(c, s, rows)
    P = c.get("prefix", 0)
    front = [rows(x, s["prefix"], P) for x in "kv"] if P else None
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["Q"].shape[:-1], dtype=torch.float64, device="cuda")
    for b, m in enumerate(s["lens"].tolist()):
        k, v = (rows(x, s["table"][b], m) for x in "kv")
        j = torch.arange(m, device="cuda")
        p = m - n + torch.arange(n, device="cuda")[:, None]
        if c["op"] == "recent":
            seen = (j <= p) & ((j < c["sinks"]) | (p - j < c["window"]))
        else:
            path = [set() for _ in range(n)]
            for t, parent in enumerate(s["parents"][b].tolist()):
                path[t] = {t} | (path[parent] if 0 <= parent < t else set())
            inside = torch.tensor([[u in x for u in range(n)] for x in path], device="cuda")
            seen = torch.ones((n, m), dtype=torch.bool, device="cuda")
            seen[:, max(0, m - n):] = inside[:, max(0, n - m):]
            seen &= p >= 0
        if front:
            k, v = torch.cat([front[0], k]), torch.cat([front[1], v])
            seen = torch.cat([seen.new_ones((n, P)), seen], 1)
        for h in range(H):
            O[b, :, h], lse[b, :, h], _ = _exact_rows(s["Q"][b, :, h].double(),
                                                      k[:, h * kv // H], v[:, h * kv // H],
                                                      seen)
    return O, lse
