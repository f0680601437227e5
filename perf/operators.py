"""The operators around a drafted tree of tokens that is served from an 8-bit paged cache: the cache's write and read,
the tree's attention over it, the tree's verification against the target's probabilities, and the move of the accepted
tokens to the front of the tree's slots.  Each in its plain form and as the framework's call, over the sizes of real use.

The model shapes are those of cdsl_inputs: 32 heads of 128 over 32 or 8 KV heads (targets), 32 of 64 over 8 (draft),
vocabularies of 32000 and 128256, trees of a root and k beams x d tokens (5 x 10, 8 x 8, 10 x 20)."""
import math

import torch

own = False

PAGE = 32


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # a prompt batch's keys and values of one layer, as the prefill writes them
        dict(name="cache 16 prompts of 256", op="cache", B=16, T=256, heads=32, hd=128, at=0, ragged=False, dtype="f32", fmt="int8"),
        # long prompts of a grouped-query model, ragged, in bf16
        dict(name="cache 24 prompts to 2047", op="cache", B=24, T=2047, heads=8, hd=128, at=0, ragged=True, dtype="bf16", fmt="e4m3"),
        # one decoded token of one prompt: latency
        dict(name="cache 1 token", op="cache", B=1, T=1, heads=8, hd=64, at=257, ragged=False, dtype="f32", fmt="int8"),
        # decoding of one token over a short prompt with the draft's heads: latency
        dict(name="attend 1 token at 256", op="attend", B=1, n=1, L=256, H=32, heads=8, hd=64, mask="tree", ragged=False, dtype="bf16", fmt="int8"),
        # decoding over long contexts: the cache's bytes
        dict(name="attend 8 tokens at 32768", op="attend", B=8, n=1, L=32768, H=32, heads=8, hd=128, mask="tree", ragged=True, dtype="bf16", fmt="int8"),
        # the 16 prompts x (root + 5 beams x 10 tokens) of a lookahead step, activations in fp32
        dict(name="attend trees of 51 at 256", op="attend", B=16, n=51, L=256, H=32, heads=32, hd=128, mask="tree", ragged=False, dtype="f32", fmt="int8"),
        # 64 prompts of 2048 tokens x (root + 8 x 8), grouped queries, ragged
        dict(name="attend trees of 65 at 2048", op="attend", B=64, n=65, L=2048, H=32, heads=8, hd=128, mask="tree", ragged=True, dtype="f32", fmt="e4m3"),
        # a chunk of a prompt over what the cache holds of it
        dict(name="attend a chunk of 509", op="attend", B=2, n=509, L=3001, H=32, heads=8, hd=128, mask="causal", ragged=True, dtype="bf16", fmt="e4m3"),
        # verification of 16 trees of 51 nodes
        dict(name="accept 16 trees of 51", op="accept", B=16, n=51, V=32000, width=5, replace=False),
        # verification of 32 trees of 65 nodes over a large vocabulary
        dict(name="accept 32 trees of 65", op="accept", B=32, n=65, V=128256, width=8, replace=True),
        # the kept path of a small tree in the draft's 16 layers: latency
        dict(name="keep 1 path of 16 layers", op="keep", B=1, n=11, L=301, heads=8, hd=64, layers=16, keep=4, fmt="e4m3"),
        # the kept paths of 16 trees in the target's 32 layers
        dict(name="keep 16 paths of 32 layers", op="keep", B=16, n=51, L=256, heads=8, hd=128, layers=32, keep=8, fmt="int8"),
    ]


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(("cache", "attend", "attend", "accept", "keep"))
    fmt, dtype = rng.choice(("int8", "e4m3")), rng.choice(("f32", "bf16"))
    heads, hd = rng.choice((1, 2, 4, 8, 8, 16, 32)), rng.choice((32, 64, 128, 128))
    if op == "cache":
        T = _log(rng, 1, 2048)
        B = _log(rng, 1, max(1, min(64, 24 * 2047 * 1024 // (T * heads * hd))))
        return dict(op=op, B=B, T=T, heads=heads, hd=hd, at=rng.randrange(0, 600), ragged=rng.random() < 0.5, dtype=dtype, fmt=fmt)
    if op == "attend":
        G = rng.choice([g for g in (1, 2, 3, 4, 5, 8) if g * heads <= 64])
        mask = rng.choice(("tree", "tree", "causal"))
        n = _log(rng, 1, 512)
        # no more (query, key) pairs and no longer a cache than the largest listed cases
        L = _log(rng, 1, min(32768, 64 * 65 * 32 * 2048 // (n * G * heads)))
        B = _log(rng, 1, max(1, min(64, 64 * 65 * 32 * 2048 // (n * G * heads * (L + n)), (8 * 32768 * 8 * 128) // ((L + n) * heads * hd))))
        return dict(op=op, B=B, n=n, L=L, H=G * heads, heads=heads, hd=hd, mask=mask, ragged=rng.random() < 0.5, dtype=dtype, fmt=fmt)
    if op == "accept":
        V = rng.choice((_log(rng, 1000, 32000), 32000, 128256, _log(rng, 32000, 131072)))
        n = _log(rng, 2, 130)
        B = _log(rng, 1, max(1, min(64, 32 * 65 * 128256 // (n * V))))
        return dict(op=op, B=B, n=n, V=V, width=rng.randrange(1, 9), replace=rng.random() < 0.5)
    n, layers = _log(rng, 2, 256), rng.randrange(1, 33)
    L = _log(rng, 1, 512)
    B = _log(rng, 1, max(1, min(32, 32 * 16 * 8 * 300 * 128 // (layers * heads * (n + L + 64) * hd))))
    return dict(op=op, B=B, n=n, L=L, heads=heads, hd=hd, layers=layers, keep=rng.randrange(1, min(n, 24) + 1), fmt=fmt)


def work(case):
    c = case
    if c["op"] == "cache":
        rows = c["B"] * c["T"] * c["heads"] * (0.5 if c["ragged"] else 1.0)
        elt = 4 if c["dtype"] == "f32" else 2
        # keys and values: read, their codes and scales written, read again, and written as values
        return {"bytes": 2 * rows * (2 * c["hd"] * elt + 2 * (c["hd"] + 4)), "flops": 2 * rows * 4 * c["hd"]}
    if c["op"] == "attend":
        share = 0.5 if c["ragged"] else 1.0  # the mean of lengths that are uniform in [0, L]
        elt = 4 if c["dtype"] == "f32" else 2
        keys = c["L"] * share + c["n"]
        seen = c["L"] * share + ((c["n"] + 1) / 2 if c["mask"] == "causal" else 1 + math.log2(c["n"]))
        return {"bytes": c["B"] * (keys * c["heads"] * (2 * c["hd"] + 8) + 2 * c["n"] * c["H"] * c["hd"] * elt),
                "flops": 4 * c["B"] * c["H"] * c["n"] * seen * c["hd"]}
    if c["op"] == "accept":
        # the two rows of the node where the walk ends
        return {"bytes": c["B"] * (8 * c["V"] + 16 * c["n"]), "flops": 3 * c["B"] * c["V"]}
    return {"bytes": 2 * c["B"] * c["layers"] * c["heads"] * c["keep"] * (2 * c["hd"] + 8), "flops": 0}


# ---------------------------------------------------------------------------
# the cache's layout.  A unit (layer, page, KV head) is 64 * hd + 256 bytes: the codes of 32 keys, those of 32 values, 32
# key scales and 32 value scales (fp32).  Codes stand in the order in which a wave's lanes take them:
#   keys    [dim / 32][(dim % 32) / 8][slot % 16][slot / 16][dim % 8]
#   values  [dim / 32][(slot % 16) / 4][dim % 16][(dim % 32) / 16][slot / 16][slot % 4]
# ---------------------------------------------------------------------------
def _unit(hd):
    return 64 * hd + 256


def _places(hd, device):
    """[32, 2 * hd + 8]: where in a unit the bytes of a slot's key, value, key scale and value scale stand."""
    s = torch.arange(PAGE, device=device)[:, None]
    d = torch.arange(hd, device=device)[None, :]
    k = d // 32 * 1024 + d % 32 // 8 * 256 + s % 16 * 16 + s // 16 * 8 + d % 8
    v = 32 * hd + d // 32 * 1024 + s % 16 // 4 * 256 + d % 16 * 16 + d % 32 // 16 * 8 + s // 16 * 4 + s % 4
    b = torch.arange(4, device=device)[None, :]
    return torch.cat([k, v, 64 * hd + 4 * s + b, 64 * hd + 128 + 4 * s + b], 1)


def _quantise(x, fmt):
    """Codes (bytes) and scales of rows x [..., hd]; quotients in 64 bits, so that values next to a border fall as they must."""
    x = x.double()
    a = x.abs().amax(-1, keepdim=True)
    tiny = 2.0 ** -126
    if fmt == "int8":
        s = (a / 127).float().double().clamp(min=tiny)
        code = torch.round(x / s)
    else:
        m, e = torch.frexp(a / 448)  # m in [0.5, 1): a power of two stays itself
        s = torch.ldexp(torch.ones_like(a), e - (m == 0.5).int())
        s = torch.where(a > 0, s, torch.zeros_like(s)).clamp(min=tiny)
        code = x / s
    bad = ~torch.isfinite(a)
    s = torch.where(bad, torch.full_like(s, math.nan), s).float()
    code = torch.where(bad, torch.zeros_like(code), code).float()
    return (code.to(torch.int8) if fmt == "int8" else code.to(torch.float8_e4m3fn)).view(torch.uint8), s[..., 0]


def _put(pool, table, K, V, at, count, fmt):
    """K, V [B, T, heads, hd] into pool [pages, heads, unit] at positions at[b] + t, t < count[b]."""
    B, T, heads, hd = K.shape
    kc, ks = _quantise(K, fmt)
    vc, vs = _quantise(V, fmt)
    row = torch.cat([kc, vc, ks[..., None].contiguous().view(torch.uint8), vs[..., None].contiguous().view(torch.uint8)], -1)
    t = torch.arange(T, device=K.device)
    pos = at[:, None].long() + t
    live = t < count[:, None]
    page = table.gather(1, (pos // PAGE).clamp(max=table.shape[1] - 1)).long()
    unit = page[..., None] * heads + torch.arange(heads, device=K.device)
    where = unit[..., None] * _unit(hd) + _places(hd, K.device)[pos % PAGE][:, :, None, :]
    pool.view(-1)[where[live]] = row[live]


def _values(pool, table, hd, fmt):
    """Keys and values [B, heads, table's tokens, hd] (fp32) of pool [pages, heads, unit]."""
    u = pool[table.long()]  # [B, P, heads, unit]
    B, P, heads, _ = u.shape
    s = u[..., 64 * hd:].contiguous().view(torch.float32).view(B, P, heads, 2, PAGE)
    kind = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    k = u[..., :32 * hd].contiguous().view(kind).view(B, P, heads, hd // 32, 4, 16, 2, 8).permute(0, 2, 1, 6, 5, 3, 4, 7)
    v = u[..., 32 * hd:64 * hd].contiguous().view(kind).view(B, P, heads, hd // 32, 4, 16, 2, 2, 4).permute(0, 2, 1, 7, 4, 8, 3, 6, 5)
    s = s.permute(3, 0, 2, 1, 4).reshape(2, B, heads, P * PAGE, 1)
    return k.reshape(B, heads, P * PAGE, hd).float() * s[0], v.reshape(B, heads, P * PAGE, hd).float() * s[1]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _rows(g, *shape):
    """Keys or values: channels of unlike sizes, as projections give them."""
    x = torch.randn(*shape, device="cuda", generator=g)
    return x * torch.exp(0.5 * torch.randn(shape[-1], device="cuda", generator=g))


def _kind(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _tree(g, B, n, width):
    """Parents [B, n] (-1 at the root, 0): node j's parent is one of the nodes shortly before it that has fewer than `width` children."""
    r = torch.rand(B, n, generator=g).tolist()
    out = []
    for b in range(B):
        par, kids = [-1], [0] * n
        for j in range(1, n):
            open_ = [i for i in range(max(0, j - 2 * width), j) if kids[i] < width] or [j - 1]
            i = open_[int(r[b][j] * len(open_))]
            kids[i] += 1
            par.append(i)
        out.append(par)
    return torch.tensor(out, dtype=torch.int32)


def _pool(g, layers, B, tokens, heads, hd):
    """A pool of pages with what earlier requests left in them, and the prompts' pages in no order."""
    per = -(-tokens // PAGE)
    pages = B * per + 3
    pool = torch.randint(0, 256, (layers, pages, heads, _unit(hd)), dtype=torch.uint8, device="cuda", generator=g)
    table = torch.randperm(pages, device="cuda", generator=g)[:B * per].view(B, per).int()
    return pool, table


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    h = torch.Generator().manual_seed(int(seed))
    ints = lambda low, high, n: torch.randint(low, high + 1, (n,), generator=h).int()  # noqa: E731
    B = c["B"]
    if c["op"] == "cache":
        count = ints(0, c["T"], B) if c["ragged"] else torch.full((B,), c["T"], dtype=torch.int32)
        at = (ints(0, c["at"], B) if c["ragged"] else torch.full((B,), c["at"], dtype=torch.int32))
        pool, table = _pool(g, 1, B, c["at"] + c["T"], c["heads"], c["hd"])
        K, V = (_rows(g, B, c["T"], c["heads"], c["hd"]).to(_kind(c["dtype"])) for _ in range(2))
        out = [torch.zeros_like(K), torch.zeros_like(V)]  # rows past a prompt's count stay as they are
        return dict(c=c, pool=pool, table=table, K=K, V=V, at=at.cuda(), count=count.cuda(), out=out)
    if c["op"] == "attend":
        n = c["n"]
        lens = ints(0, c["L"], B) if c["ragged"] else torch.full((B,), c["L"], dtype=torch.int32)
        lens[B // 2] = c["L"]
        pool, table = _pool(g, 1, B, c["L"] + n, c["heads"], c["hd"])
        for b in range(B):
            T = int(lens[b]) + n
            K, V = (_rows(g, 1, T, c["heads"], c["hd"]) for _ in range(2))
            for t in range(0, T, 4096):
                part = slice(t, min(T, t + 4096))
                _put(pool[0], table[b:b + 1], K[:, part], V[:, part], torch.tensor([t], device="cuda"),
                     torch.tensor([part.stop - t], device="cuda"), c["fmt"])
        q = (1.5 * torch.randn(B, n, c["H"], c["hd"], device="cuda", generator=g)).to(_kind(c["dtype"]))
        parents = _tree(h, B, n, 4).cuda() if c["mask"] == "tree" else None
        return dict(c=c, pool=pool, table=table, q=q, lens=lens.cuda(), longest=int(lens.max()), parents=parents)
    if c["op"] == "accept":
        n, V = c["n"], c["V"]
        parents = _tree(h, B, n, c["width"])
        z = torch.empty(B, n, V, device="cuda").normal_(0, 2.5, generator=g)
        p = torch.softmax(z, -1)
        z += torch.empty(B, n, V, device="cuda").normal_(0, 0.7, generator=g)
        q = torch.softmax(z, -1)
        del z
        most = min(V, 8)
        drawn = torch.multinomial(q.view(-1, V), most, replacement=c["replace"], generator=g).view(B, n, most)
        rank = torch.zeros(B, n, dtype=torch.long)
        for b, par in enumerate(parents.tolist()):
            seen = [0] * n
            for j in range(1, n):
                rank[b, j] = seen[par[j]] % most
                seen[par[j]] += 1
        par = parents.clamp(min=0).long().cuda()
        tokens = drawn.gather(1, par[..., None].expand(B, n, most)).gather(2, rank.cuda()[..., None])[..., 0].int()
        u, v = torch.rand(B, n, device="cuda", generator=g), torch.rand(B, device="cuda", generator=g)
        return dict(c=c, p=p, q=q, tokens=tokens.contiguous(), parents=parents.cuda(), u=u, v=v)
    n = c["n"]
    lens = torch.full((B,), c["L"], dtype=torch.int32)
    pool, table = _pool(g, c["layers"], B, c["L"] + n, c["heads"], c["hd"])
    path = torch.full((B, n), -1, dtype=torch.int32)
    for b in range(B):
        path[b, :c["keep"]] = torch.cat([torch.zeros(1, dtype=torch.long), 1 + torch.randperm(n - 1, generator=h)[:c["keep"] - 1].sort().values]).int()
    count = ints(1, c["keep"], B)
    count[0] = c["keep"]
    return dict(c=c, pool=pool, table=table, lens=lens.cuda(), path=path.cuda(), count=count.cuda())


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    c = state["c"]
    if own:
        return _own(state)
    if c["op"] == "cache":
        return _plain_cache(state)
    if c["op"] == "attend":
        return _plain_attend(state)
    if c["op"] == "accept":
        return _plain_accept(state)
    return _plain_keep(state)


def _own(state):
    from paper_2412_10418_amd import binding as bd

    c = state["c"]
    if c["op"] == "accept":
        return bd.cdsl_op_tree_accept(state["p"], state["q"], state["tokens"], state["parents"], state["u"], state["v"], replace=c["replace"])
    cache = bd.QuantCache(state["pool"], state["table"], c["hd"], c["fmt"])
    if c["op"] == "cache":
        bd.cdsl_op_kvq_write(cache, state["K"], state["V"], start=state["at"], count=state["count"])
        return bd.cdsl_op_kvq_read(cache, c["T"], start=state["at"], count=state["count"], out=state["out"])
    if c["op"] == "attend":
        return bd.cdsl_op_tree_attention(cache, state["q"], state["lens"], state["parents"], max_len=state["longest"])
    return bd.cdsl_op_kvq_keep(cache, state["lens"], state["path"], state["count"]), state["pool"]


def _plain_cache(s):
    c = s["c"]
    _put(s["pool"][0], s["table"], s["K"], s["V"], s["at"], s["count"], c["fmt"])
    t = torch.arange(c["T"], device="cuda")
    at = (s["at"][:, None].long() + t).clamp(max=s["table"].shape[1] * PAGE - 1)
    live = (t < s["count"][:, None])[:, :, None, None]
    for out, x in zip(s["out"], _values(s["pool"][0], s["table"], c["hd"], c["fmt"])):
        rows = x.transpose(1, 2).gather(1, at[:, :, None, None].expand(-1, -1, c["heads"], c["hd"]))
        out.copy_(torch.where(live, rows.to(out.dtype), out))
    return s["out"]


def _ancestors(parents):
    """[B, n, n]: whether node j is i or above i."""
    B, n = parents.shape
    up = torch.eye(n, device=parents.device).repeat(B, 1, 1)
    j = torch.arange(n, device=parents.device)
    up = ((parents[:, :, None] == j) | (j[:, None] == j)).float()
    for _ in range(max(1, (n - 1).bit_length())):
        up = (up @ up).clamp(max=1)
    return up > 0


def _plain_attend(s):
    c, q = s["c"], s["q"]
    B, n, H, hd = q.shape
    heads = c["heads"]
    K, V = _values(s["pool"][0], s["table"], hd, c["fmt"])
    at = torch.arange(K.shape[2], device="cuda") - s["lens"][:, None]  # [B, tokens]: the node at a position
    if s["parents"] is None:
        node = at[:, None, :] <= torch.arange(n, device="cuda")[:, None]
    else:
        node = _ancestors(s["parents"]).gather(2, at.clamp(0, n - 1).long()[:, None, :].expand(B, n, -1))
    sees = ((at < 0)[:, None, :] | (node & (at < n)[:, None, :]))[:, None, :, None, :]
    held = (at < n)[:, None, :, None]
    K, V = torch.where(held, K, torch.zeros_like(K)), torch.where(held, V, torch.zeros_like(V))
    x = q.float().view(B, n, heads, H // heads, hd).permute(0, 2, 1, 3, 4).reshape(B, heads, -1, hd)
    z = (x @ K.transpose(2, 3).contiguous() / math.sqrt(hd)).view(B, heads, n, H // heads, -1)
    z = torch.where(sees, z, torch.full_like(z, -math.inf))
    w = torch.exp(z - z.amax(-1, keepdim=True))
    o = (w.view(B, heads, -1, w.shape[-1]) @ V).view(B, heads, n, H // heads, hd) / w.sum(-1, keepdim=True)
    return o.permute(0, 2, 1, 3, 4).reshape(B, n, H, hd).to(q.dtype)


def _plain_accept(s):
    """The walk in 64 bits: node j is tested while its parent is the node reached; a rejection leaves what the target's
    probabilities have above the draft's."""
    p, q, tokens, parents, u = s["p"], s["q"], s["tokens"].long(), s["parents"], s["u"].double()
    B, n, V = p.shape
    b = torch.arange(B, device="cuda")
    at = torch.zeros(B, dtype=torch.long, device="cuda")
    P, Q = p[:, 0].double(), q[:, 0].double()
    rest, over = torch.ones_like(u[:, 0]), torch.zeros(B, dtype=torch.bool, device="cuda")
    path = torch.full((B, n), -1, dtype=torch.int32, device="cuda")
    path[:, 0] = 0
    length = torch.ones(B, dtype=torch.long, device="cuda")
    for j in range(1, n):
        x = tokens[:, j]
        test = (parents[:, j] == at) & (rest > 0) & ~over
        px, qx = P[b, x], Q[b, x] / rest
        took = test & (u[:, j] * qx <= px) & (px > 0)
        fell = test & ~took
        R = (P - Q / rest[:, None]).clamp(min=0)
        Z = R.sum(1)
        over = over | (fell & (Z <= 0))
        P = torch.where((fell & (Z > 0))[:, None], R / Z[:, None], P)
        if not s["c"]["replace"]:
            rest = torch.where(fell, rest - Q[b, x], rest)
            Q[b, x] = torch.where(fell, torch.zeros_like(qx), Q[b, x])
        P = torch.where(took[:, None], p[:, j].double(), P)
        Q = torch.where(took[:, None], q[:, j].double(), Q)
        rest = torch.where(took, torch.ones_like(rest), rest)
        at = torch.where(took, torch.full_like(at, j), at)
        path[b, length.clamp(max=n - 1)] = torch.where(took, torch.full_like(path[:, 0], j), path[b, length.clamp(max=n - 1)])
        length = length + took
    sums = P.cumsum(1)
    last = torch.where(P > 0, torch.arange(V, device="cuda"), -1).amax(1)
    drawn = torch.minimum((sums <= (s["v"].double() * sums[:, -1])[:, None]).sum(1), last)
    token = torch.where(over, p[b, at].argmax(1), drawn)
    return path, length.int(), token.int()


def _plain_keep(s):
    c, pool = s["c"], s["pool"]
    heads, hd = c["heads"], c["hd"]
    i = torch.arange(c["n"], device="cuda")
    live = i < s["count"][:, None]

    def where(pos):
        page = s["table"].gather(1, pos // PAGE).long()
        unit = page[..., None] * heads + torch.arange(heads, device="cuda")
        return (unit[..., None] * _unit(hd) + _places(hd, "cuda")[pos % PAGE][:, :, None, :])[live].view(-1)

    L = s["lens"][:, None].long()
    flat = pool.view(c["layers"], -1)
    flat[:, where(L + i)] = flat[:, where(L + s["path"].clamp(min=0))]
    return s["lens"] + s["count"], pool


# ---------------------------------------------------------------------------
# what the definitions give in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] in ("accept", "keep"):
        return None  # tokens, nodes, lengths and bytes: whole values
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "cache":
        out = []
        for x, o in zip((s["K"], s["V"]), s["out"]):
            x = x.to(torch.float64)
            top = x.abs().max(dim=-1, keepdim=True).values
            if c["fmt"] == "int8":
                step = torch.clamp((top / 127).to(torch.float32).to(torch.float64), min=2.0 ** -126)
                y = torch.round(x / step) * step
            else:
                step = torch.clamp(torch.exp2(torch.ceil(torch.log2(top / 448))), min=2.0 ** -126)
                mag = (x / step).abs()
                grain = torch.exp2(torch.floor(torch.log2(mag.clamp(min=2.0 ** -6))) - 3)  # four bits, subnormal below 2^-6
                y = torch.sign(x) * torch.round(mag / grain) * grain * step
            rows = torch.arange(c["T"], device=x.device)[None, :] < s["count"][:, None]
            out.append(torch.where(rows[:, :, None, None], y, o.to(torch.float64)))
        return out
    B, n, H, hd = s["q"].shape
    heads, G = c["heads"], H // c["heads"]
    signed = torch.arange(256).to(torch.uint8).view(torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn).to(torch.float64).cuda()
    at = _places(hd, "cuda")
    out = torch.empty(B, n, H, hd, dtype=torch.float64, device="cuda")
    for b in range(B):
        L = int(s["lens"][b])
        pos = torch.arange(L + n, device="cuda")
        unit = s["pool"][0][s["table"][b].long()[pos // PAGE]]  # [tokens, heads, unit]
        byte = unit.gather(2, at[pos % PAGE][:, None, :].expand(-1, heads, -1))
        scale = byte[..., 2 * hd:].contiguous().view(torch.float32).to(torch.float64)
        K = signed[byte[..., :hd].long()] * scale[..., :1]
        V = signed[byte[..., hd:2 * hd].long()] * scale[..., 1:]
        see = torch.ones(n, L + n, dtype=torch.bool)
        if s["parents"] is None:
            see[:, L:] = torch.ones(n, n).tril().bool()
        else:
            par, up = s["parents"][b].tolist(), torch.zeros(n, n, dtype=torch.bool)
            for i in range(n):
                if par[i] >= 0:
                    up[i] = up[par[i]]
                up[i, i] = True
            see[:, L:] = up
        see = see.cuda()
        for h in range(heads):
            x = s["q"][b, :, h * G:(h + 1) * G].to(torch.float64)  # [n, G, hd]
            z = torch.matmul(x, K[:, h].t().contiguous()) / math.sqrt(hd)
            z = z.masked_fill(~see[:, None, :], -math.inf)
            w = torch.exp(z - z.max(dim=-1, keepdim=True).values)
            out[b, :, h * G:(h + 1) * G] = torch.matmul(w, V[:, h].contiguous()) / w.sum(-1, keepdim=True)
    return out
