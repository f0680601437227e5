"""The operators of serving from a paged cache that is held in 4 bits and whose pages are shared: the cache's write, read
and kept path, the attention of trees, chunks and single tokens over it, and the pages' forking, reserving, freeing,
compacting and copying.  Each in its plain form and as the framework's call, over the sizes of real use.

The model shapes are those of cdsl_inputs: 32 heads of 128 over 32 or 8 KV heads (targets), 32 of 64 over 8 (draft),
16 or 32 layers, trees of a root and k beams x d tokens."""
import math

import torch

own = False

PAGE = 32
NONE = 1 << 40


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # long prompts of a grouped-query model, ragged, as the prefill writes them, and read back
        dict(name="cache 24 prompts to 2047", op="cache", B=24, T=2047, heads=8, hd=128, at=0, ragged=True, dtype="bf16"),
        # one decoded token of one prompt: latency
        dict(name="cache 1 token", op="cache", B=1, T=1, heads=8, hd=64, at=257, ragged=False, dtype="f32"),
        # the kept paths of 16 trees in the target's 32 layers
        dict(name="keep 16 paths of 32 layers", op="keep", B=16, n=51, L=256, heads=8, hd=128, layers=32, keep=8),
        # decoding of one token over a short prompt with the draft's heads: latency
        dict(name="attend 1 token at 256", op="attend", B=1, n=1, L=256, H=32, heads=8, hd=64, mask="tree", ragged=False, dtype="bf16"),
        # decoding over long contexts: the cache's bytes
        dict(name="attend 8 tokens at 32768", op="attend", B=8, n=1, L=32768, H=32, heads=8, hd=128, mask="tree", ragged=True, dtype="bf16"),
        # 64 prompts of 2048 tokens x (root + 8 x 8), grouped queries, ragged, activations in fp32
        dict(name="attend trees of 65 at 2048", op="attend", B=64, n=65, L=2048, H=32, heads=8, hd=128, mask="tree", ragged=True, dtype="f32"),
        # a chunk of a prompt over what the cache holds of it
        dict(name="attend a chunk of 509", op="attend", B=2, n=509, L=3001, H=32, heads=8, hd=128, mask="causal", ragged=True, dtype="bf16"),
        # the 8 beams of 8 prompts go on from the chosen one: its pages are shared, the last one copied in all layers
        dict(name="beams 8 x 8 at 500", op="beams", B=8, k=8, winners=1, L=500, T=8, heads=8, hd=128, layers=32, fmt="mxfp4"),
        # 4 beams of one prompt in the draft's 16 layers: latency
        dict(name="beams 1 x 4 at 100", op="beams", B=1, k=4, winners=4, L=100, T=1, heads=8, hd=64, layers=16, fmt="mxfp4"),
        # a serving batch: a third of the prompts has ended and others take their rows, the rest goes on by a token
        dict(name="turnover of 256 prompts", op="turnover", B=256, P=257, pages=20011, L=2047, layers=1, heads=1, hd=32, fmt="e4m3"),
        # a pool whose requests left holes: the used pages to the front
        dict(name="compact 512 pages", op="compact", B=24, P=33, pages=512, layers=16, heads=8, hd=128, fmt="mxfp4", used=0.5),
        # pages of prefilled prompts to another pool
        dict(name="copy 130 pages", op="copy", n=130, pages=300, layers=32, heads=8, hd=128, fmt="mxfp4"),
    ]


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(("cache", "cache", "keep", "attend", "attend", "attend", "attend", "beams", "beams", "turnover", "compact", "copy"))
    fmt, dtype = rng.choice(("mxfp4", "mxfp4", "int8", "e4m3")), rng.choice(("f32", "bf16"))
    heads, hd = rng.choice((1, 2, 4, 8, 8, 16, 32)), rng.choice((32, 64, 128, 128))
    layers = rng.randrange(1, 33)
    page = layers * heads * _unit(hd, fmt)
    if op == "cache":
        T = _log(rng, 1, 2048)
        B = _log(rng, 1, max(1, min(64, 24 * 2047 * 1024 // (2 * T * heads * hd))))
        return dict(op=op, B=B, T=T, heads=heads, hd=hd, at=rng.randrange(0, 600), ragged=rng.random() < 0.5, dtype=dtype)
    if op == "attend":
        G = rng.choice([g for g in (1, 2, 3, 4, 5, 8) if g * heads <= 64])
        mask = rng.choice(("tree", "tree", "causal"))
        n = _log(rng, 1, 512)
        # no more (query, key) pairs and no longer a cache than the largest listed cases
        L = _log(rng, 1, min(32768, 64 * 65 * 32 * 2048 // (2 * n * G * heads)))
        B = _log(rng, 1, max(1, min(64, 64 * 65 * 32 * 2048 // (2 * n * G * heads * (L + n)), (8 * 32768 * 8 * 128) // ((L + n) * heads * hd))))
        return dict(op=op, B=B, n=n, L=L, H=G * heads, heads=heads, hd=hd, mask=mask, ragged=rng.random() < 0.5, dtype=dtype)
    if op == "keep":
        n = _log(rng, 2, 256)
        L = _log(rng, 1, 512)
        B = _log(rng, 1, max(1, min(32, 32 * 16 * 8 * 300 * 128 // (layers * heads * (n + L + 64) * hd))))
        return dict(op=op, B=B, n=n, L=L, heads=heads, hd=hd, layers=layers, keep=rng.randrange(1, min(n, 24) + 1))
    if op == "beams":
        L, k = _log(rng, 1, 2048), rng.randrange(2, 11)
        T = rng.randrange(1, 41)
        B = _log(rng, 1, max(1, min(16, 220_000_000 // (page * (L // PAGE + 2 + 3 * k)))))
        return dict(op=op, B=B, k=k, winners=rng.randrange(1, k + 1), L=L, T=T, heads=heads, hd=hd, layers=layers, fmt=fmt)
    if op == "turnover":
        B, L = _log(rng, 1, 256), _log(rng, 1, 2047)
        need = B * (L // PAGE + 2)
        return dict(op=op, B=B, P=L // PAGE + 2 + rng.randrange(0, 200), pages=_log(rng, need // 2 + 2, 2 * need + 40), L=L, layers=1, heads=1, hd=32, fmt=fmt)
    pages = _log(rng, 3, max(3, min(2000, 250_000_000 // page)))
    if op == "compact":
        B = _log(rng, 1, 64)
        return dict(op=op, B=B, P=2 * pages // B + 2, pages=pages, layers=layers, heads=heads, hd=hd, fmt=fmt, used=rng.uniform(0.2, 0.9))
    return dict(op=op, n=_log(rng, 1, max(1, pages // 2)), pages=pages, layers=layers, heads=heads, hd=hd, fmt=fmt)


def work(case):
    c = case
    if c["op"] == "cache":
        rows = c["B"] * c["T"] * c["heads"] * (0.5 if c["ragged"] else 1.0)
        elt = 4 if c["dtype"] == "f32" else 2
        # keys and values: read, their codes and scales written, read again, and written as values
        return {"bytes": 2 * rows * c["hd"] * (2 * elt + 2 * 17 / 32), "flops": 2 * rows * 4 * c["hd"]}
    if c["op"] == "attend":
        share = 0.5 if c["ragged"] else 1.0  # the mean of lengths that are uniform in [0, L]
        elt = 4 if c["dtype"] == "f32" else 2
        keys = c["L"] * share + c["n"]
        seen = c["L"] * share + ((c["n"] + 1) / 2 if c["mask"] == "causal" else 1 + math.log2(c["n"]))
        return {"bytes": c["B"] * (keys * c["heads"] * c["hd"] * 17 / 16 + 2 * c["n"] * c["H"] * c["hd"] * elt),
                "flops": 4 * c["B"] * c["H"] * c["n"] * seen * c["hd"]}
    if c["op"] == "keep":
        return {"bytes": 2 * c["B"] * c["layers"] * c["heads"] * c["keep"] * c["hd"] * 17 / 16, "flops": 0}
    page = c["layers"] * c["heads"] * _unit(c["hd"], c["fmt"])
    if c["op"] == "beams":
        k, w = c["k"], c["winners"]
        copies = c["B"] * (k - w * (1 - (1 - 1 / w) ** k)) * 31 / 32  # beams less the parents that were drawn
        return {"bytes": 2 * copies * page + 8 * c["B"] * k * (c["L"] // PAGE + 1), "flops": 0}
    if c["op"] == "turnover":
        # the tables and the counts once, and what changes in them
        return {"bytes": 4 * c["B"] * c["P"] + 4 * c["pages"] + 8 * c["B"] * c["L"] // (3 * PAGE), "flops": 0}
    if c["op"] == "compact":
        return {"bytes": 2 * c["pages"] * c["used"] * (1 - c["used"]) * page + 8 * c["B"] * c["P"] + 8 * c["pages"], "flops": 0}
    return {"bytes": 2 * c["n"] * page, "flops": 0}


# ---------------------------------------------------------------------------
# the cache's layout.  A unit (layer, page, KV head) is 34 * hd bytes: the codes of 32 keys, those of 32 values, the scales
# of the keys and those of the values.  A byte holds the codes of two dims (the lower 4 bits the even one), a scale byte x
# counts 2^(x - 127) for 32 dims of a token, 255 NaN.  They stand in the order in which a wave's lanes take them
# (of dim / 32 % 2 only what there is):
#   keys          [dim / 64][(dim % 32) / 8][slot % 16][dim / 32 % 2][slot / 16][dim % 8 / 2]
#   values        [dim / 64][(slot % 16) / 4][dim % 32 / 2][dim / 32 % 2][slot / 16][slot % 4]
#   key scales    [dim / 64][slot % 16][dim / 32 % 2][slot / 16]
#   value scales  [dim / 64][(slot % 16) / 4][dim / 32 % 2][slot / 16][slot % 4]
# ---------------------------------------------------------------------------
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _unit(hd, fmt="mxfp4"):
    return 34 * hd if fmt == "mxfp4" else 64 * hd + 256


def _places(hd, device):
    """[32, hd + hd / 16]: where in a unit the bytes of a slot's key, value, key scales and value scales stand."""
    W = min(hd, 64) // 32
    s = torch.arange(PAGE, device=device)[:, None]
    d = 2 * torch.arange(hd // 2, device=device)[None, :]
    z = 32 * torch.arange(hd // 32, device=device)[None, :]
    k = d // 64 * 1024 + (d % 32 // 8 * 16 + s % 16) * 8 * W + d // 32 % 2 * 8 + s // 16 * 4 + d % 8 // 2
    v = 16 * hd + d // 64 * 1024 + (s % 16 // 4 * 16 + d % 32 // 2) * 8 * W + d // 32 % 2 * 8 + s // 16 * 4 + s % 4
    ks = 32 * hd + z // 64 * 64 + s % 16 * 2 * W + z // 32 % 2 * 2 + s // 16
    vs = 33 * hd + z // 64 * 64 + s % 16 // 4 * 8 * W + z // 32 % 2 * 8 + s // 16 * 4 + s % 4
    return torch.cat([k, v, ks, vs], 1)


def _quantise(x):
    """Code bytes [..., hd / 2] and scale bytes [..., hd / 32] of rows x [..., hd]."""
    x = x.double()
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    x = torch.where(bad, torch.zeros_like(x), x).clamp(-1.5 * 2.0 ** 127, 1.5 * 2.0 ** 127).unflatten(-1, (-1, 32))
    a = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(a / 6)  # m in [0.5, 1): a power of two stays itself
    e = torch.where(a > 0, e - (m == 0.5).int(), torch.full_like(e, -125)).clamp(min=-125)
    r = x.abs() / torch.ldexp(torch.ones_like(a), e)
    step = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0))
    r = torch.round(r / step) * step
    code = torch.where(r <= 2, 2 * r, torch.where(r <= 4, r + 2, torch.full_like(r, 7))) + 8 * torch.signbit(x)
    code = code.flatten(-2).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, torch.where(bad, torch.full_like(e[..., 0], 255), e[..., 0] + 127).to(torch.uint8)


def _put(pool, table, K, V, at, count):
    """K, V [B, T, heads, hd] into pool [pages, heads, unit] at positions at[b] + t, t < count[b]."""
    B, T, heads, hd = K.shape
    kc, ks = _quantise(K)
    vc, vs = _quantise(V)
    row = torch.cat([kc, vc, ks, vs], -1)
    t = torch.arange(T, device=K.device)
    pos = at[:, None].long() + t
    live = t < count[:, None]
    page = table.gather(1, (pos // PAGE).clamp(max=table.shape[1] - 1)).long()
    unit = page[..., None] * heads + torch.arange(heads, device=K.device)
    where = unit[..., None] * _unit(hd) + _places(hd, K.device)[pos % PAGE][:, :, None, :]
    pool.view(-1)[where[live]] = row[live]


def _values(pool, table, hd):
    """Keys and values [B, heads, table's tokens, hd] (fp32) of pool [pages, heads, unit]."""
    u = pool[table.long()]  # [B, P, heads, unit]
    B, P, heads, _ = u.shape
    W = min(hd, 64) // 32
    C = hd // 32 // W
    grid = torch.tensor(GRID + tuple(-x for x in GRID), device=pool.device)
    nibbles = lambda b: grid[torch.stack([b & 15, b >> 4], -1).int()]  # noqa: E731
    power = lambda b: torch.where(b == 255, math.nan, torch.ldexp(torch.ones_like(b, dtype=torch.float32), b.int() - 127))  # noqa: E731
    k = nibbles(u[..., :16 * hd]).view(B, P, heads, C, 4, 16, W, 2, 4, 2).permute(0, 2, 1, 7, 5, 3, 6, 4, 8, 9)
    v = nibbles(u[..., 16 * hd:32 * hd]).view(B, P, heads, C, 4, 16, W, 2, 4, 2).permute(0, 2, 1, 7, 4, 8, 3, 6, 5, 9)
    ks = power(u[..., 32 * hd:33 * hd]).view(B, P, heads, C, 16, W, 2).permute(0, 2, 1, 6, 4, 3, 5)
    vs = power(u[..., 33 * hd:]).view(B, P, heads, C, 4, W, 2, 4).permute(0, 2, 1, 6, 4, 7, 3, 5)
    shape = (B, heads, P * PAGE, hd // 32)
    return ((k.reshape(*shape, 32) * ks.reshape(*shape, 1)).view(B, heads, P * PAGE, hd),
            (v.reshape(*shape, 32) * vs.reshape(*shape, 1)).view(B, heads, P * PAGE, hd))


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


def _bytes(g, *shape):
    return torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=g)


def _pool(g, layers, B, tokens, heads, hd):
    """A pool of pages with what earlier requests left in them, and the prompts' pages in no order."""
    per = -(-tokens // PAGE)
    pages = B * per + 3
    return _bytes(g, layers, pages, heads, _unit(hd)), torch.randperm(pages, device="cuda", generator=g)[:B * per].view(B, per).int()


def _counts(table, pages):
    """How many entries of a table hold each page."""
    return torch.bincount(table[table >= 0].long().flatten(), minlength=pages).int()


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    h = torch.Generator().manual_seed(int(seed))
    ints = lambda low, high, *n: torch.randint(low, high + 1, n, generator=h).int()  # noqa: E731
    B = c.get("B", 1)
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
                     torch.tensor([part.stop - t], device="cuda"))
        q = (1.5 * torch.randn(B, n, c["H"], c["hd"], device="cuda", generator=g)).to(_kind(c["dtype"]))
        parents = _tree(h, B, n, 4).cuda() if c["mask"] == "tree" else None
        return dict(c=c, pool=pool, table=table, q=q, lens=lens.cuda(), longest=int(lens.max()), parents=parents)
    if c["op"] == "keep":
        n = c["n"]
        lens = torch.full((B,), c["L"], dtype=torch.int32)
        pool, table = _pool(g, c["layers"], B, c["L"] + n, c["heads"], c["hd"])
        path = torch.full((B, n), -1, dtype=torch.int32)
        for b in range(B):
            path[b, :c["keep"]] = torch.cat([torch.zeros(1, dtype=torch.long), 1 + torch.randperm(n - 1, generator=h)[:c["keep"] - 1].sort().values]).int()
        count = ints(1, c["keep"], B)
        count[0] = c["keep"]
        return dict(c=c, pool=pool, table=table, lens=lens.cuda(), path=path.cuda(), count=count.cuda())
    unit = _unit(c["hd"], c["fmt"])
    if c["op"] == "beams":
        # every beam has the prompt's whole pages and a last one of its own; the pool has as many free ones again
        k, whole, more = c["k"], c["L"] // PAGE, c["T"] // PAGE + 2
        pages = B * (whole + k * 2 * more)
        order = torch.randperm(pages, generator=h).int()
        table = torch.full((B, k, whole + more), -1, dtype=torch.int32)
        table[:, :, :whole] = order[:B * whole].view(B, 1, whole)
        table[:, :, whole] = order[B * whole:B * (whole + k)].view(B, k)
        parents = (ints(0, c["winners"] - 1, B, k) + torch.arange(B)[:, None] * k).int()
        lens = torch.full((B * k,), c["L"], dtype=torch.int32)
        pool = _bytes(g, c["layers"], pages, c["heads"], unit)
        refs = _counts(table, pages)
        count = torch.full_like(lens, c["T"])
        return dict(c=c, pool=pool, table=table.view(B * k, -1).cuda(), refs=refs.cuda(), parents=parents.view(-1).cuda(), lens=lens.cuda(), count=count.cuda())
    if c["op"] == "turnover":
        # the first two pages are one system prompt's, shared by all that are long enough
        P, pages = c["P"], c["pages"]
        lens = ints(0, c["L"], B)
        held = (lens + PAGE - 1) // PAGE
        i = torch.arange(P)
        has = (i < held[:, None]) & ~((i < 2) & (lens[:, None] >= 2 * PAGE))
        rank = (has.flatten().cumsum(0) - 1).view(B, P)
        order = torch.randperm(pages, generator=h).int()
        table = torch.where(has & (rank < pages - 2), order[2 + rank.clamp(0, pages - 3)], -1)
        table[:, :2] = torch.where(lens[:, None] >= 2 * PAGE, order[:2], table[:, :2])[:, :P]
        left = torch.where(torch.rand(B, generator=h) < 1 / 3, 0, lens)  # 0: it has ended
        count = torch.where(left == 0, ints(1, c["L"], B), 1)
        table = table.int().contiguous()
        pool = _bytes(g, c["layers"], pages, c["heads"], unit)
        return dict(c=c, pool=pool, table=table.cuda(), refs=_counts(table, pages).cuda(), left=left.int().cuda(), count=count.int().cuda())
    if c["op"] == "compact":
        # each used page in one to three tables
        P, pages = c["P"], c["pages"]
        used = torch.randperm(pages, generator=h)[:max(1, round(pages * c["used"]))].int()
        held = torch.cat([used, used[:len(used) // 3], used[:len(used) // 9]])[:B * P]
        table = torch.full((B * P,), -1, dtype=torch.int32)
        table[torch.randperm(B * P, generator=h)[:len(held)]] = held
        refs = _counts(table, pages)
        start = torch.cat([table, refs]).cuda()
        now = start.clone()
        pool = _bytes(g, c["layers"], pages, c["heads"], unit)
        return dict(c=c, pool=pool, start=start, now=now, table=now[:B * P].view(B, P), refs=now[B * P:])
    src, dst = (torch.randperm(c["pages"], generator=h)[:c["n"]].int() for _ in range(2))
    pool, other = (_bytes(g, c["layers"], c["pages"], c["heads"], unit) for _ in range(2))
    return dict(c=c, pool=pool, other=other, table=torch.zeros(1, 1, dtype=torch.int32, device="cuda"), src=src.cuda(), dst=dst.cuda())


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    s, op = state, state["c"]["op"]
    if own:
        return _own(s)
    if op == "cache":
        return _plain_cache(s)
    if op == "attend":
        return _plain_attend(s)
    if op == "keep":
        return _plain_keep(s)
    if op == "beams":
        _plain_fork(s["table"], s["refs"], s["parents"])
        got = _plain_reserve(s["pool"], s["table"], s["refs"], s["lens"], s["count"], s["c"]["T"])
        return got, s["table"], s["refs"], s["pool"]
    if op == "turnover":
        _plain_free(s["table"], s["refs"], s["left"])
        return _plain_reserve(s["pool"], s["table"], s["refs"], s["left"], s["count"], s["c"]["L"]), s["table"], s["refs"]
    if op == "compact":
        s["now"].copy_(s["start"])  # the holes again
        return _plain_compact(s["pool"], s["table"], s["refs"]), s["table"], s["refs"], s["pool"]
    s["other"][:, s["dst"].long()] = s["pool"][:, s["src"].long()]
    return s["other"]


def _own(s):
    from paper_2412_10418_amd import binding as bd

    c = s["c"]
    cache = bd.QuantCache(s["pool"], s["table"], c["hd"], c.get("fmt", "mxfp4"))
    if c["op"] == "cache":
        bd.cdsl_op_kvq_write(cache, s["K"], s["V"], start=s["at"], count=s["count"])
        return bd.cdsl_op_kvq_read(cache, c["T"], start=s["at"], count=s["count"], out=s["out"])
    if c["op"] == "attend":
        return bd.cdsl_op_tree_attention(cache, s["q"], s["lens"], s["parents"], max_len=s["longest"])
    if c["op"] == "keep":
        return bd.cdsl_op_kvq_keep(cache, s["lens"], s["path"], s["count"]), s["pool"]
    if c["op"] == "beams":
        bd.cdsl_op_pages_fork(cache, s["refs"], s["parents"])
        got = bd.cdsl_op_pages_reserve(cache, s["refs"], s["lens"], s["count"], c["T"])
        return got, s["table"], s["refs"], s["pool"]
    if c["op"] == "turnover":
        bd.cdsl_op_pages_free(cache, s["refs"], s["left"])
        return bd.cdsl_op_pages_reserve(cache, s["refs"], s["left"], s["count"], c["L"]), s["table"], s["refs"]
    if c["op"] == "compact":
        s["now"].copy_(s["start"])  # the holes again
        return bd.cdsl_op_pages_compact(cache, s["refs"]), s["table"], s["refs"], s["pool"]
    bd.cdsl_op_pages_copy(cache, s["src"], bd.QuantCache(s["other"], s["table"], c["hd"], c["fmt"]), s["dst"])
    return s["other"]


def _plain_cache(s):
    c = s["c"]
    _put(s["pool"][0], s["table"], s["K"], s["V"], s["at"], s["count"])
    t = torch.arange(c["T"], device="cuda")
    at = (s["at"][:, None].long() + t).clamp(max=s["table"].shape[1] * PAGE - 1)
    live = (t < s["count"][:, None])[:, :, None, None]
    K, V = _values(s["pool"][0], s["table"], c["hd"])
    at = at[:, :, None, None].expand(-1, -1, c["heads"], c["hd"])
    s["out"][0].copy_(torch.where(live, K.transpose(1, 2).gather(1, at).to(s["K"].dtype), s["out"][0]))
    s["out"][1].copy_(torch.where(live, V.transpose(1, 2).gather(1, at).to(s["V"].dtype), s["out"][1]))
    return s["out"]


def _doubled(up, times):
    """The relation `up` followed 2^times times."""
    return up if times == 0 else _doubled((up @ up).clamp(max=1), times - 1)


def _ancestors(parents):
    """[B, n, n]: whether node j is i or above i."""
    n = parents.shape[1]
    j = torch.arange(n, device=parents.device)
    up = ((parents[:, :, None] == j) | (j[:, None] == j)).float()
    return _doubled(up, max(1, (n - 1).bit_length())) > 0


def _plain_attend(s):
    c, q = s["c"], s["q"]
    B, n, H, hd = q.shape
    heads = c["heads"]
    K, V = _values(s["pool"][0], s["table"], hd)
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


def _holds(refs, ids, by):
    """Adds `by` for each entry of ids that holds a page to its count."""
    held = (ids >= 0) & (ids < refs.shape[0])
    refs.index_add_(0, torch.where(held, ids, 0).long().flatten(), torch.where(held, by, 0).int().flatten())


def _plain_fork(table, refs, parents):
    new = table[parents.long()]
    _holds(refs, table, -1)
    _holds(refs, new, 1)
    table.copy_(new)


def _plain_free(table, refs, lens):
    drop = torch.arange(table.shape[1], device="cuda") * PAGE >= lens[:, None]
    _holds(refs, torch.where(drop, table, -1), -1)
    table.masked_fill_(drop, -1)


def _plain_reserve(pool, table, refs, lens, count, T):
    """Pages of their own for count[b] tokens behind the lens[b] that prompt b has: where an entry has none, and where the
    page is shared, unless the others that hold it leave it in the same call (the first of them keeps it).  They are the
    lowest free ones, in the order of the prompts and their pages; a shared page with tokens in it is copied."""
    (B, P), pages = table.shape, refs.shape[0]
    M = -(-T // PAGE) + 1
    i = lens[:, None].long() // PAGE + torch.arange(M, device="cuda")
    in_run = (count > 0)[:, None] & (i * PAGE < (lens + count)[:, None])
    touched = in_run & (i < P)
    ids = table.gather(1, i.clamp(max=P - 1)).long()
    page = ids.clamp(min=0)
    R = refs[page]
    held = touched & (ids >= 0)
    shared = held & (R > 1)
    e = torch.arange(B * M, device="cuda").view(B, M)
    at = torch.where(shared, page, pages).flatten()
    leave = torch.zeros(pages + 1, dtype=torch.int32, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    first = torch.full((pages + 1,), NONE, device="cuda").scatter_reduce_(0, at, e.flatten(), "amin")
    keeps = shared & (leave[page] == R) & (first[page] == e)
    need = (touched & ~held) | (shared & ~keeps)
    number = (need.flatten().cumsum(0) - 1).view(B, M)
    free = refs == 0
    room = free.sum()
    lowest = torch.argsort(~free, stable=True)
    given = need & (number < room)
    last = torch.full((pages + 1,), -1, device="cuda").scatter_reduce_(0, at, torch.where(need, number, -1).flatten(), "amax")
    keeps &= last[page] < room
    new = lowest[number.clamp(0, pages - 1)]
    moved = given & shared
    copied = moved & (i * PAGE < lens[:, None])
    pool[:, new[copied]] = pool[:, page[copied]]
    table[e[given] // M, i[given]] = new[given].int()
    refs[new[given]] = 1
    _holds(refs, torch.where(moved, ids, -1), -1)
    fine = (given | keeps | (held & ~shared)).int().cumprod(1).sum(1)
    return torch.minimum(count, ((lens // PAGE + fine) * PAGE - lens).clamp(min=0)).int()


def _plain_compact(pool, table, refs):
    """The highest used page to the lowest free one, and so on, until the used ones are the first."""
    used = refs > 0
    n = used.sum()
    ids = torch.arange(refs.shape[0], device="cuda")
    dst, src = ids[~used & (ids < n)], ids[used & (ids >= n)].flip(0)
    to = ids.index_copy(0, src, dst)
    pool[:, dst] = pool[:, src]
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
    refs[dst] = refs[src]
    refs[src] = 0
    return n.int()


# ---------------------------------------------------------------------------
# what the definitions give in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] not in ("cache", "attend"):
        return None  # pages, lengths and bytes: whole values
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "cache":
        out = []
        for x, o in zip((s["K"], s["V"]), s["out"]):
            x = x.to(torch.float64)
            block = x.reshape(*x.shape[:-1], c["hd"] // 32, 32)
            top = block.abs().max(dim=-1, keepdim=True).values
            unit = torch.clamp(torch.exp2(torch.ceil(torch.log2(top / 6))), min=2.0 ** -125)
            mag = (block / unit).abs()
            grain = torch.exp2(torch.floor(torch.log2(mag.clamp(min=1.0))) - 1)  # two bits, subnormal below 1
            y = (torch.sign(block) * torch.round(mag / grain) * grain * unit).reshape(x.shape)
            rows = torch.arange(c["T"], device=x.device)[None, :] < s["count"][:, None]
            out.append(torch.where(rows[:, :, None, None], y, o.to(torch.float64)))
        return out
    B, n, H, hd = s["q"].shape
    heads, G = c["heads"], H // c["heads"]
    code = torch.arange(16, dtype=torch.float64)
    mag = torch.where(code % 8 < 2, code % 2 / 2, (1 + code % 2 / 2) * 2.0 ** (code % 8 // 2 - 1))
    value = torch.where(code < 8, mag, -mag).cuda()
    at = _places(hd, "cuda")
    out = torch.empty(B, n, H, hd, dtype=torch.float64, device="cuda")
    for b in range(B):
        L = int(s["lens"][b])
        pos = torch.arange(L + n, device="cuda")
        unit = s["pool"][0][s["table"][b].long()[pos // PAGE]]  # [tokens, heads, unit]
        byte = unit.gather(2, at[pos % PAGE][:, None, :].expand(-1, heads, -1)).long()

        def rows(codes, scales):
            y = torch.stack([value[codes % 16], value[codes // 16]], -1).reshape(len(pos), heads, hd // 32, 32)
            return (y * torch.exp2(scales.to(torch.float64) - 127)[..., None]).reshape(len(pos), heads, hd)

        K, V = rows(byte[..., :hd // 2], byte[..., hd:hd + hd // 32]), rows(byte[..., hd // 2:hd], byte[..., hd + hd // 32:])
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
