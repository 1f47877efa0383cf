"""Timed cases of the operators around a paged 4-bit key/value cache, each with a plain form.

  rope    the norm of every query and key head and the position rotation, in one pass
  write   new keys and values quantised into the pages, the accepted path published, entries read back
  attn    decode attention of every tree node over the pages (a tree of one node is plain decoding)
  pages   page bookkeeping of a batch: fork a prompt into several continuations, or retire half of the
          requests, compact the pool and admit others

Keys and values are held as e2m1 numbers (4 bits) in blocks of 16 along the head, each block with an e4m3 scale
(8 bits).  One page holds, for every KV head, first the keys and then the values of its positions: all codes
([position, 64 bytes], even elements in the low half of a byte), then all scales ([position, 8 bytes]).

With ``own`` false ``run`` computes everything with elementary torch operations; with ``own`` true it makes the calls
that a user of the library makes.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_DH = 128
_SPINE = 12          # longest principal chain of a "spine" tree
_DEEPEST = 16        # no tree here is deeper
_P_STOP = 0.35       # accepted lengths: P(L = l) = p (1 - p)^(l - 1), cut at the leaf
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _rope(B, N, **kw):
    c = dict(kind="rope", B=B, N=N, Hq=32, Hkv=8, dh=_DH, rot=_DH, style="half", axes=1, turns=False, far=16384, dtype="bf16")
    c.update(kw)
    return c


def _cache(kind, B, N, ctx, **kw):
    c = dict(kind=kind, B=B, N=N, rows=N, Hq=32, Hkv=8, ctx=ctx, page=64, shape="spine", depth=min(_SPINE, N))
    c.update(kw)
    return c


def listed() -> List[dict]:
    return [
        # one request decoding one token: the smallest call, launches and latency only
        dict(_rope(1, 1), name="rope b1 n1"),
        # the tree of a serving batch: 28 nodes a request, positions from the tree itself
        dict(_rope(8, 28), name="rope b8 n28"),
        # a long prompt of a model that reads pictures: three position axes, half of each head rotated, 8192 tokens
        dict(_rope(1, 8192, rot=64, axes=3, turns=True, far=131072), name="rope 8k tokens 3 axes"),
        # one cycle of a serving batch: the tree's entries written, the accepted path published and read back
        dict(_cache("write", 8, 28, 16384, rows=32), name="write tree b8 n28"),
        # a prompt's keys and values into the cache
        dict(_cache("write", 1, 8191, 0, page=128, shape="prompt", depth=1), name="write prompt 8k"),
        # one chat request, one token
        dict(_cache("attn", 1, 1, 4000), name="attn b1 n1 ctx4k"),
        # a decoding batch without drafts
        dict(_cache("attn", 16, 1, 16384), name="attn b16 n1 ctx16k"),
        # short trees (a few drafts a request) on small pages
        dict(_cache("attn", 4, 8, 8192, rows=8, page=16, depth=4), name="attn b4 n8 ctx8k"),
        # the verifier's batch of coding-agent requests of uneven length
        dict(_cache("attn", 8, 28, 16384, rows=32), name="attn b8 n28 ctx16k"),
        # one request at full context with a large tree
        dict(_cache("attn", 1, 64, 131072, rows=64, page=128, shape="random", depth=8), name="attn b1 n64 ctx128k"),
        # eight prompts continued eight ways each: pages shared, the page being written copied, recurrent states copied
        dict(kind="pages", what="fork", R=8, ways=8, ctx=8000, add=32, Hkv=8, page=64, layers=16, states=2, Hv=32, name="pages fork 8 x 8"),
        # half of the requests leave and others come, twice: the pool is compacted in between
        dict(kind="pages", what="turnover", R=32, ways=1, ctx=1000, add=0, Hkv=8, page=64, layers=8, states=0, Hv=0, name="pages turnover 32"),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _tree_of(rng: random.Random, N: int):
    if N > 1 and rng.random() < 0.5:
        depth = rng.randint(4, 12)
        while sum(2 ** k for k in range(1, depth + 1)) < N:
            depth += 1
        return "random", depth
    return "spine", max(1, min(N, rng.randint(2, _SPINE)))


def draw(rng: random.Random) -> dict:
    kind = rng.choice(["rope", "rope", "write", "write", "attn", "attn", "attn", "attn", "pages", "pages"])
    page = rng.choice([16, 32, 64, 64, 128])
    if kind == "rope":
        Hkv = rng.choice([1, 2, 4, 8])
        heads = dict(Hkv=Hkv, Hq=Hkv * rng.choice([1, 2, 4, 4, 8]), dh=rng.choice([64, 128, 128]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                     style=rng.choice(["half", "half", "pairs"]), far=_log_int(rng, 64, 1 << 20))
        heads["rot"] = heads["dh"] // rng.choice([1, 1, 2, 4])
        if rng.random() < 0.5:     # trees
            return _rope(_log_int(rng, 1, 32), _log_int(rng, 1, 64), **heads)
        top = 8192 * 40 * 128 // ((heads["Hq"] + heads["Hkv"]) * heads["dh"] * (2 if heads["dtype"] == "f32" else 1))
        axes = rng.choice([1, 3])
        return _rope(1, _log_int(rng, 65, min(top, 8192)), axes=axes, turns=axes == 3 and rng.random() < 0.5, **heads)
    if kind == "write":
        Hkv = rng.choice([1, 2, 4, 8])
        if rng.random() < 0.4:
            return _cache("write", 1, _log_int(rng, 65, 8191), 0, Hkv=Hkv, Hq=4 * Hkv, page=page, shape="prompt", depth=1)
        N = _log_int(rng, 1, 64)
        shape, depth = _tree_of(rng, N)
        return _cache("write", _log_int(rng, 1, 16), N, _log_int(rng, 1, 16384), Hkv=Hkv, Hq=4 * Hkv, page=page, shape=shape, depth=depth,
                      rows=N + (-N % 32 if rng.random() < 0.5 else 0))
    if kind == "attn":
        Hkv = rng.choice([2, 4, 8, 8])
        B, N = _log_int(rng, 1, 16), 1 if rng.random() < 0.4 else _log_int(rng, 2, 64)
        shape, depth = _tree_of(rng, N)
        G = rng.choice([1, 2, 4, 4, 8])
        top = min(131072, 262144 // B, 131072 * 64 * 4 // (B * N * G))
        return _cache("attn", B, N, _log_int(rng, 1, top), Hq=G * Hkv, Hkv=Hkv, page=page, shape=shape, depth=depth,
                      rows=N + (-N % 32 if rng.random() < 0.5 else 0))
    if rng.random() < 0.5:
        R, ways = _log_int(rng, 1, 8), _log_int(rng, 1, 8)
        return dict(kind="pages", what="fork", R=R, ways=ways, ctx=_log_int(rng, 1, 8000), add=_log_int(rng, 1, 256), Hkv=rng.choice([2, 4, 8]),
                    page=page if page < 128 else 64, layers=_log_int(rng, 1, 16), states=rng.choice([0, 1, 2]), Hv=rng.choice([8, 16, 32]))
    return dict(kind="pages", what="turnover", R=2 * _log_int(rng, 1, 16), ways=1, ctx=_log_int(rng, 16, 1000), add=0, Hkv=rng.choice([2, 4, 8]),
                page=page if page < 128 else 64, layers=_log_int(rng, 1, 8), states=0, Hv=0)


# ---------------------------------------------------------------------------
# trees and paths, on the host
# ---------------------------------------------------------------------------
def _tree(rng: random.Random, shape: str, N: int, depth: int) -> List[int]:
    """parent[i] in {-1} U [0, i); -1 is the committed context."""
    if shape == "spine":   # a principal chain; two siblings per level; the rest lengthens those branches
        s = max(1, min(depth, (N + 1) // 2))
        parent = [i - 1 for i in range(s)]
        tails = []
        for lvl in range(s):
            for _ in range(2):
                if len(parent) < N:
                    parent.append(lvl - 1)
                    tails.append((len(parent) - 1, lvl + 1))
        j = 0
        while len(parent) < N:
            node, dep = tails[j % len(tails)]
            parent.append(node if dep < depth + 3 else rng.randrange(-1, s))
            tails[j % len(tails)] = (len(parent) - 1, dep + 1) if dep < depth + 3 else (parent[-1], dep)
            j += 1
        return parent
    while True:            # frontier expansion, fan-out U{1..4}
        parent, dep, frontier = [], [], [-1]
        while len(parent) < N and frontier:
            p = frontier.pop(rng.randrange(len(frontier)))
            d = 0 if p < 0 else dep[p]
            if d >= depth:
                continue
            for _ in range(rng.randint(1, 4)):
                if len(parent) < N:
                    parent.append(p)
                    dep.append(d + 1)
                    frontier.append(len(parent) - 1)
        if len(parent) == N:
            return parent


def _ancestors(parent: List[int], i: int) -> List[int]:
    path = []
    while i >= 0:
        path.append(i)
        i = parent[i]
    return path[::-1]


def _accepted(rng: random.Random, parent: List[int]) -> List[int]:
    """A walk from the root along uniformly drawn children, of geometric length."""
    kids: Dict[int, List[int]] = {}
    for i, p in enumerate(parent):
        kids.setdefault(p, []).append(i)
    n = 1
    while rng.random() >= _P_STOP:
        n += 1
    path, cur = [], -1
    while len(path) < n and kids.get(cur):
        cur = rng.choice(kids[cur])
        path.append(cur)
    return path


def _plan(case: dict, seed: int) -> dict:
    """Trees, slot maps, accepted paths and context lengths of one batch."""
    rng = random.Random(seed * 7919 + 17)
    B, N, rows = case["B"], case["N"], case.get("rows", case["N"])
    parents = [_tree(rng, case.get("shape", "spine"), N, case.get("depth", min(_SPINE, N))) for _ in range(B)]
    slot = np.array([rng.sample(range(rows), N) if rows > N else list(range(N)) for _ in range(B)], dtype=np.int32)
    anc = [[_ancestors(p, i) for i in range(N)] for p in parents]
    depth = np.array([[len(a) for a in row] for row in anc], dtype=np.int32)
    vis = np.zeros((B, N, rows), dtype=bool)
    for b in range(B):
        for i in range(N):
            vis[b, i, slot[b, anc[b][i]]] = True
    paths = [_accepted(rng, p) for p in parents]
    lmax = int(depth.max())
    acc = np.full((B, lmax), -1, dtype=np.int32)
    for b, p in enumerate(paths):
        acc[b, :len(p)] = p
    return dict(parent=np.array(parents, dtype=np.int32), slot_h=slot, rng=rng, lmax=lmax, slot=torch.from_numpy(slot).cuda(),
                depth=torch.from_numpy(depth).cuda(), vis=torch.from_numpy(vis).cuda(), accepted=torch.from_numpy(acc).cuda(),
                length=torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda"))


class _Draws:
    """Seeded tensors drawn on the device."""

    def __init__(self, seed: int):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape, dt=torch.float32, std=1.0):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, std, generator=self.g)

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, dtype=torch.int32, device="cuda", generator=self.g)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


_contexts: Dict[int, object] = {}


def _ctx():
    """One context per device, kept for the life of the process, as a server keeps it."""
    from paper_2609_23900_b200 import binding
    dev = torch.cuda.current_device()
    if dev not in _contexts:
        _contexts[dev] = binding.Context(dev)
    return _contexts[dev]


# ---------------------------------------------------------------------------
# rope
# ---------------------------------------------------------------------------
def _sections(case: dict) -> List[int]:
    """Frequency pairs of the time, height and width axes."""
    n = case["rot"] // 2
    side = n * 3 // 8 if not case["turns"] else n // 3
    return [n - 2 * side, side, side]


def _axis_of(case: dict) -> List[int]:
    n, (a, b, c) = case["rot"] // 2, _sections(case)
    if case["axes"] == 1:
        return [0] * n
    if case["turns"]:      # t, h, w, t, h, w, ... as long as height and width have pairs left
        return [j % 3 if j % 3 and j // 3 < b else 0 for j in range(n)]
    return [0] * a + [1] * b + [2] * c


def _prepare_rope(case: dict, seed: int) -> dict:
    r, dt, dh, T = _Draws(seed), _DT[case["dtype"]], case["dh"], case["B"] * case["N"]
    Hq, Hkv = case["Hq"], case["Hkv"]
    qkv = r.normal(T, (Hq + 2 * Hkv) * dh, dt=dt, std=2.0)          # the projection's output: q and k are parts of its rows
    s = dict(q=qkv[:, :Hq * dh].unflatten(1, (Hq, dh)), k=qkv[:, Hq * dh:(Hq + Hkv) * dh].unflatten(1, (Hkv, dh)),
             q_weight=(1.0 + r.normal(dh, std=0.2)).to(dt), k_weight=(1.0 + r.normal(dh, std=0.2)).to(dt), eps=1e-6,
             inv_freq=(1e6 ** (-torch.arange(case["rot"] // 2, dtype=torch.float64) * 2 / case["rot"])).float().cuda(),
             axis=torch.tensor(_axis_of(case), device="cuda"), q_out=torch.empty(T, Hq, dh, dtype=dt, device="cuda"),
             k_out=torch.empty(T, Hkv, dh, dtype=dt, device="cuda"))
    if case["N"] <= 64:    # trees: a node's position is its context's length and its depth
        p = _plan(case, seed)
        s["ctx_len"] = r.ints(case["far"] // 2, case["far"], case["B"])
        s["depth"] = p["depth"]
    else:
        p = None
        start = case["far"] - T if case["far"] > T else 0
        t = start + torch.arange(T, dtype=torch.int32, device="cuda")
        s["pos"] = torch.stack([t] + [r.ints(0, 64, T) for _ in range(case["axes"] - 1)])
    if own:
        from paper_2609_23900_b200 import binding
        s["desc"] = _ctx().tree_desc(p["parent"]) if p else None
        s["layer"] = binding.QkNormRope(q=s["q"], k=s["k"], q_out=s["q_out"], k_out=s["k_out"], inv_freq=s["inv_freq"], q_weight=s["q_weight"],
                                        k_weight=s["k_weight"], eps=s["eps"], style=case["style"], pos=s.get("pos"), ctx_len=s.get("ctx_len"),
                                        sections=_sections(case) if case["axes"] == 3 else None, turns=case["turns"])
    return s


def _rope_plain(x, weight, eps, cos, sin, style, out):
    rot = 2 * cos.shape[-1]
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + eps) * weight.float()
    a, b = (y[..., :rot // 2], y[..., rot // 2:rot]) if style == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([u, v], dim=-1) if style == "half" else torch.stack([u, v], dim=-1).flatten(-2)
    out.copy_(torch.cat([turned, y[..., rot:]], dim=-1))


def _run_rope(s: dict):
    if own:
        _ctx().qk_norm_rope(s["layer"], s["desc"])
        return {"q": s["q_out"], "k": s["k_out"]}
    pos = s["pos"] if "pos" in s else (s["ctx_len"][:, None] + s["depth"] - 1).reshape(1, -1)
    angle = (pos.double()[s["axis"]] * s["inv_freq"].double()[:, None]).T[:, None, :]          # far positions: 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()
    _rope_plain(s["q"], s["q_weight"], s["eps"], cos, sin, s["case"]["style"], s["q_out"])
    _rope_plain(s["k"], s["k_weight"], s["eps"], cos, sin, s["case"]["style"], s["k_out"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _exact_rope(case: dict, s: dict):
    """The definition pair by pair: complex numbers turned by exp(i angle)."""
    n = case["rot"] // 2
    pos = (s["pos"] if "pos" in s else (s["ctx_len"][:, None] + s["depth"] - 1).reshape(1, -1)).cpu().numpy().astype(np.float64)
    freq = s["inv_freq"].cpu().numpy().astype(np.float64)
    turn = np.stack([np.exp(1j * pos[a] * f) for a, f in zip(_axis_of(case), freq)], axis=1)     # [T, n]
    got = {}
    for name in ("q", "k"):
        x = s[name].double().cpu().numpy()
        y = x / np.sqrt((x * x).sum(-1, keepdims=True) / case["dh"] + s["eps"]) * s[name + "_weight"].double().cpu().numpy()
        first, second = (slice(0, n), slice(n, 2 * n)) if case["style"] == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
        z = (y[..., first] + 1j * y[..., second]) * turn[:, None, :]
        y[..., first], y[..., second] = z.real, z.imag
        got[name] = y
    return got


# ---------------------------------------------------------------------------
# the 4-bit cache
# ---------------------------------------------------------------------------
def _quantise(x: torch.Tensor):
    """x [..., 128] -> codes [..., 64] and scales [..., 8], both as bytes.  A block's scale is its largest magnitude over 6, rounded to
    e4m3; a code is the nearest e2m1 number to value over scale, ties to the even code.  (Comparing the value with a border times the scale
    is exact: bf16 values, and borders times scales of at most seven bits.)"""
    b = x.float().unflatten(-1, (8, 16))
    scale = (b.abs().amax(dim=-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    y, s = b.abs(), scale.float()[..., None]
    code = ((y > 0.25 * s).to(torch.uint8) + (y >= 0.75 * s) + (y > 1.25 * s) + (y >= 1.75 * s) + (y > 2.5 * s) + (y >= 3.5 * s) + (y > 5.0 * s))
    code = torch.where(s > 0, code, torch.zeros_like(code)) | ((b < 0).to(torch.uint8) << 3)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.view(torch.uint8)


def _values(codes: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    """codes [..., 64], scales [..., 8] -> fp32 values [..., 128] (exact)."""
    table = torch.tensor(_E2M1 + [-v for v in _E2M1], device=codes.device)
    e = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    return (table[e.int()].unflatten(-1, (8, 16)) * scales.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _parts(pages: torch.Tensor, page: int):
    """Views of a pool [n_pages, Hkv, 2, page * 72]: codes [.., page, 64] and scales [.., page, 8]."""
    return pages[..., :page * 64].unflatten(-1, (page, 64)), pages[..., page * 64:].unflatten(-1, (page, 8))


def _prepare_cache(case: dict, seed: int) -> dict:
    r, B, N, P, Hkv = _Draws(seed), case["B"], case["N"], case["page"], case["Hkv"]
    prompt = case["shape"] == "prompt"
    p = None if prompt else _plan(case, seed)
    rng = random.Random(seed * 31 + 5) if prompt else p["rng"]
    suffix = N if prompt else case["rows"]
    ctx = [case["ctx"] if b == 0 else rng.randint((case["ctx"] + 1) // 2, case["ctx"]) for b in range(B)]          # uneven requests
    per_row = -(-(case["ctx"] + suffix) // P)
    n_pages = (B + 1) * per_row + 3
    order = torch.randperm(n_pages, device="cuda", generator=r.g).to(torch.int32)
    table = order[:(B + 1) * per_row].reshape(B + 1, per_row).clone()
    rows = list(range(B + 1))
    rng.shuffle(rows)
    pages = torch.empty(n_pages, Hkv, 2, P * 72, dtype=torch.uint8, device="cuda")
    codes, scales = _parts(pages, P)
    c, q = _quantise(r.normal(n_pages, Hkv, 2, P, _DH, dt=torch.bfloat16))
    codes.copy_(c)
    scales.copy_(q)
    s = dict(plan=p, table=table, pages=pages, ctx_len=_i32(ctx), row=_i32(rows[:B]), ctx_host=ctx,
             status=torch.full((B,), -1, dtype=torch.int32, device="cuda"))
    if case["kind"] == "attn":
        s.update(q=r.normal(B, N, case["Hq"], _DH, dt=torch.bfloat16), out=torch.empty(B, N, case["Hq"], _DH, dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty(B, N, case["Hq"], device="cuda"))
    else:
        s.update(k_new=r.normal(B, N, Hkv, _DH, dt=torch.bfloat16, std=2.0), v_new=r.normal(B, N, Hkv, _DH, dt=torch.bfloat16))
        if prompt:
            s.update(tok_row=s["row"].expand(N).contiguous(), tok_pos=torch.arange(N, dtype=torch.int32, device="cuda"))
        else:              # read back: the published path and what follows it, up to the deepest tree's length
            back = min(N, _DEEPEST)
            s.update(tok_row=s["row"][:, None].expand(B, back).reshape(-1).contiguous(),
                     tok_pos=(s["ctx_len"][:, None] + torch.arange(back, dtype=torch.int32, device="cuda")).reshape(-1),
                     ctx_len_out=torch.zeros_like(s["ctx_len"]))
        T = s["tok_row"].numel()
        s.update(k_back=torch.empty(T, Hkv, _DH, dtype=torch.bfloat16, device="cuda"), v_back=torch.empty(T, Hkv, _DH, dtype=torch.bfloat16, device="cuda"))
    if own:
        from paper_2609_23900_b200 import binding
        s["desc"] = None if prompt else _ctx().tree_desc(p["parent"], slot=p["slot_h"], n_slots=case["rows"])
        kw = {n: s[n] for n in ("q", "out", "lse", "k_new", "v_new") if n in s}
        if case["kind"] == "attn":
            kw["work"] = torch.empty(_ctx().kv4_work_bytes(s["desc"], case["Hq"], Hkv), dtype=torch.uint8, device="cuda")
        s["layer"] = binding.Kv4Layer(Hq=case["Hq"], Hkv=Hkv, pages=pages, table=table, page_size=P, scale=_DH ** -0.5, ctx_len=s["ctx_len"],
                                      cache_row=s["row"], status=s["status"], **kw)
        s["packed"] = _ctx().pack_kv4([s["layer"]])
    return s


def _run_write(s: dict):
    case, P = s["case"], s["case"]["page"]
    prompt = case["shape"] == "prompt"
    if own:
        c = _ctx()
        if prompt:
            c.kv4_append(s["packed"], s["tok_row"], s["tok_pos"])
        else:
            c.kv4_write_tree(s["desc"], s["packed"])
            c.kv4_publish(s["desc"], s["packed"], s["plan"]["accepted"], s["plan"]["length"], s["ctx_len_out"])
        c.kv4_read(s["layer"], s["tok_row"], s["tok_pos"], s["k_back"], s["v_back"])
        return {"k": s["k_back"], "v": s["v_back"], **({} if prompt else {"ctx_len": s["ctx_len_out"]})}
    codes, scales = _parts(s["pages"], P)
    c, q = _quantise(torch.stack([s["k_new"], s["v_new"]], dim=3))                     # [B, N, Hkv, 2, ...]
    if prompt:
        row, pos = s["tok_row"].reshape(1, -1), s["tok_pos"].reshape(1, -1)
    else:
        row, pos = s["row"][:, None], s["ctx_len"][:, None] + s["plan"]["slot"]
    place = s["table"][row, pos // P].long(), pos.long() % P
    codes[place[0], :, :, place[1]] = c
    scales[place[0], :, :, place[1]] = q
    if not prompt:         # the accepted path to its new places, all reads first
        p, t = s["plan"], torch.arange(s["plan"]["lmax"], device="cuda")
        taken = t < p["length"][:, None]
        node = torch.where(taken, p["accepted"], 0).long()
        a = s["ctx_len"][:, None] + torch.where(taken, torch.gather(p["slot"], 1, node), t)
        b = (s["ctx_len"][:, None] + t)
        src, dst = (s["table"][row, a // P].long(), a.long() % P), (s["table"][row, b // P].long(), b.long() % P)
        c, q = codes[src[0], :, :, src[1]], scales[src[0], :, :, src[1]]
        codes[dst[0], :, :, dst[1]] = c
        scales[dst[0], :, :, dst[1]] = q
        torch.add(s["ctx_len"], p["length"], out=s["ctx_len_out"])
    page, at = s["table"][s["tok_row"], s["tok_pos"] // P].long(), s["tok_pos"].long() % P
    kv = _values(codes[page, :, :, at], scales[page, :, :, at])                         # [T, Hkv, 2, 128]
    s["k_back"].copy_(kv[:, :, 0])
    s["v_back"].copy_(kv[:, :, 1])
    return {"k": s["k_back"], "v": s["v_back"], **({} if prompt else {"ctx_len": s["ctx_len_out"]})}


def _exact_write(case: dict, s: dict):
    """Entry by entry: the entry that the publication leaves at each place, quantised in 64 bits by search among all numbers."""
    P, Hkv = case["page"], case["Hkv"]
    e4m3 = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()       # 0 .. 448, ascending
    e2m1 = np.array(_E2M1)

    def nearest(x, grid):  # ties to the even place in the grid
        i = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
        lo, hi = x - grid[i - 1], grid[i] - x
        return np.where((lo < hi) | ((lo == hi) & ((i - 1) % 2 == 0)), i - 1, i)

    def held(x):           # [T, Hkv, 128] -> the values the cache stands for
        b = x.reshape(*x.shape[:-1], 8, 16)
        sc = e4m3[nearest(np.abs(b).max(-1) / 6, e4m3)][..., None]
        mag = e2m1[nearest(np.divide(np.abs(b), sc, out=np.zeros_like(b), where=sc > 0), e2m1)]
        return (np.sign(b) * mag * sc).reshape(x.shape)

    new = {n: held(s[n + "_new"].double().cpu().numpy().reshape(-1, Hkv, _DH)) for n in ("k", "v")}
    if case["shape"] == "prompt":
        return {**new}
    p, B, N = s["plan"], case["B"], case["N"]
    acc, ln, slot, table, rows = (t.cpu().numpy() for t in (p["accepted"], p["length"], p["slot"], s["table"], s["row"]))
    codes, scales = (v.cpu().numpy() for v in _parts(s["pages"], P))
    back = min(N, _DEEPEST)
    got = {n: np.zeros((B, back, Hkv, _DH)) for n in ("k", "v")}
    sign = np.array(_E2M1 + [-v for v in _E2M1])
    byte = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    for b in range(B):
        at = {int(slot[b, i]): i for i in range(N)}
        for t in range(back):
            node = int(acc[b, t]) if t < ln[b] else at.get(t)
            for w, n in enumerate(("k", "v")):
                if node is not None:
                    got[n][b, t] = new[n][b * N + node]
                else:      # a place that no node was written to: what the cache held
                    pos = s["ctx_host"][b] + t
                    pg = table[rows[b], pos // P]
                    c = codes[pg, :, w, pos % P]
                    v = sign[np.stack([c & 15, c >> 4], axis=-1).reshape(Hkv, _DH)]
                    got[n][b, t] = v * np.repeat(byte[scales[pg, :, w, pos % P]], 16, axis=-1)
    return {"k": got["k"].reshape(-1, Hkv, _DH), "v": got["v"].reshape(-1, Hkv, _DH), "ctx_len": None}


def _run_attn(s: dict):
    if own:
        _ctx().kv4_attention(s["desc"], s["packed"])
        return {"out": s["out"], "lse": s["lse"]}
    case, p, P = s["case"], s["plan"], s["case"]["page"]
    B, N, Hq, Hkv, S = case["B"], case["N"], case["Hq"], case["Hkv"], case["ctx"] + case["rows"]
    codes, scales = _parts(s["pages"][s["table"][s["row"]]], P)                         # [B, pages, Hkv, 2, P, ...]
    order = (0, 2, 3, 1, 4, 5)
    kv = _values(codes.permute(order).flatten(3, 4), scales.permute(order).flatten(3, 4))[:, :, :, :S]     # [B, Hkv, 2, S, 128]
    G = Hq // Hkv
    q = s["q"].float().reshape(B, N, Hkv, G, _DH).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * N, _DH)
    logits = (q @ kv[:, :, 0].transpose(-1, -2)) * _DH ** -0.5
    at = torch.arange(S, device="cuda") - s["ctx_len"][:, None]                         # slot of each position; below 0: context
    inside = (at >= 0) & (at < case["rows"])
    seen = torch.gather(p["vis"], 2, at.clamp(0, case["rows"] - 1)[:, None, :].expand(B, N, S)) & inside[:, None, :] | (at < 0)[:, None, :]
    logits.unflatten(2, (G, N)).masked_fill_(~seen[:, None, None], -math.inf)
    m = logits.amax(dim=-1, keepdim=True)
    w = torch.exp(logits.sub_(m))
    total = w.sum(dim=-1, keepdim=True)
    out = (w @ kv[:, :, 1]) / total
    back = lambda t: t.unflatten(2, (G, N)).permute(0, 3, 1, 2, 4).reshape(B, N, Hq, -1)  # noqa: E731
    s["out"].copy_(back(out))
    s["lse"].copy_(back(m + total.log()).squeeze(-1))
    return {"out": s["out"], "lse": s["lse"]}


def _exact_attn(case: dict, s: dict):
    """Sequence by sequence and head by head in 64 bits, each node over its own list of positions."""
    p, P, G = s["plan"], case["page"], case["Hq"] // case["Hkv"]
    B, N = case["B"], case["N"]
    out, lse = np.zeros((B, N, case["Hq"], _DH)), np.zeros((B, N, case["Hq"]))
    number = torch.tensor(_E2M1 + [-v for v in _E2M1], dtype=torch.float64, device="cuda")
    row, slot = s["row"].tolist(), p["slot_h"]
    for b in range(B):
        ctx, mine = s["ctx_host"][b], s["pages"][s["table"][row[b]].long()]
        for h in range(case["Hkv"]):
            kv = []
            for w in range(2):
                raw = mine[:, h, w]
                c, f = raw[:, :P * 64].reshape(-1, 64), raw[:, P * 64:].reshape(-1, 8).view(torch.float8_e4m3fn).double()
                v = torch.empty(c.shape[0], _DH, dtype=torch.float64, device="cuda")
                v[:, 0::2], v[:, 1::2] = number[(c % 16).long()], number[(c // 16).long()]
                kv.append(v * f.repeat_interleave(16, dim=1))
            k, v = kv
            tail = torch.full((N, case["rows"]), -math.inf, dtype=torch.float64, device="cuda")
            for i in range(N):
                tail[i, [int(slot[b, a]) for a in _ancestors(p["parent"][b].tolist(), i)]] = 0.0
            for g in range(G):
                x = s["q"][b, :, h * G + g].double() @ k[:ctx + case["rows"]].T / math.sqrt(_DH)
                x[:, ctx:] += tail
                z = torch.logsumexp(x, dim=1)
                lse[b, :, h * G + g] = z.cpu().numpy()
                out[b, :, h * G + g] = (torch.exp(x - z[:, None]) @ v[:ctx + case["rows"]]).cpu().numpy()
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------
# pages
# ---------------------------------------------------------------------------
def _prepare_pages(case: dict, seed: int) -> dict:
    r, rng, P, R, ways = _Draws(seed), random.Random(seed * 7919 + 17), case["page"], case["R"], case["ways"]
    fork = case["what"] == "fork"
    lens = [case["ctx"] if i == 0 else rng.randint((case["ctx"] + 1) // 2, case["ctx"]) for i in range(R)]
    held = [-(-n // P) for n in lens]
    n_rows = R * (1 + ways) + 1 if fork else R + 1
    max_pages = -(-(case["ctx"] + case["add"]) // P) + 1
    spare = R * ways * (-(-case["add"] // P) + 2) if fork else 0
    n_pages = R * held[0] + spare + 5
    order = torch.randperm(n_pages, device="cuda", generator=r.g).to(torch.int32)
    rows = list(range(n_rows))
    rng.shuffle(rows)
    table = torch.full((n_rows, max_pages), -1, dtype=torch.int32, device="cuda")
    row_pages = [0] * n_rows
    at = 0
    for row, n in zip(rows, held):
        table[row, :n] = order[at:at + n]
        row_pages[row] = n
        at += n
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[order[:at].long()] = 1
    free_list = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free_list[:n_pages - at] = order[at:]
    nbytes = case["Hkv"] * 2 * P * 72
    pools = [torch.randint(0, 256, (n_pages, nbytes), dtype=torch.uint8, device="cuda", generator=r.g) for _ in range(case["layers"])]
    s = dict(table=table, row_pages=_i32(row_pages), refs=refs, free_list=free_list, free_count=_i32([n_pages - at]), pools=pools)
    if fork:
        kids = rows[R:R + R * ways]
        s.update(src=_i32([rows[i] for i in range(R) for _ in range(ways)]), dst=_i32(kids), start=_i32([lens[i] for i in range(R) for _ in range(ways)]),
                 states=[r.normal(n_rows, case["Hv"], _DH, _DH) for _ in range(case["states"])])
    else:
        half = R // 2
        s.update(rows_a=_i32(rows[:half]), rows_b=_i32(rows[half:R]), len_a=_i32(lens[:half]), len_b=_i32(lens[half:]))
    if own:
        from paper_2609_23900_b200 import binding
        s["pt"] = binding.PageTable(page_size=P, table=table, row_pages=s["row_pages"], refs=refs, free_list=free_list, free_count=s["free_count"],
                                    pools=pools, work=torch.empty(binding.pages_work_ints(n_rows, n_pages), dtype=torch.int32, device="cuda"))
        if fork and case["states"]:
            s["state_rows"] = binding.RowBlocks(s["states"])
    return s


def _free(s: dict, rows, P):
    """All pages of the rows given back: the last one listed goes onto the list first."""
    rows = rows.long()
    mine = torch.arange(s["table"].shape[1], device="cuda") < s["row_pages"][rows][:, None]
    page = s["table"][rows][mine].long()
    s["refs"].index_add_(0, page, torch.full_like(page, -1, dtype=torch.int32))
    event = torch.arange(page.numel(), device="cuda")
    first = torch.full_like(s["refs"], 1 << 30, dtype=torch.int64).scatter_reduce_(0, page, event, "amin")
    back = page[(s["refs"][page] == 0) & (first[page] == event)].flip(0)
    n = s["free_count"].long()
    s["free_list"][n + torch.arange(back.numel(), device="cuda")] = back.to(torch.int32)
    s["free_count"] += back.numel()
    s["table"][rows] = -1
    s["row_pages"][rows] = 0


def _reserve(s: dict, rows, start, end, P):
    """Positions [start, end) of the rows made writable: shared pages among them are replaced by copies (the last listed sharer keeps the page
    when all of its sharers are listed), missing ones are added; new pages come off the list's end, a row's copies before its additions."""
    rows, idx = rows.long(), torch.arange(s["table"].shape[1], device="cuda")
    have, need = s["row_pages"][rows][:, None], -(-end // P)[:, None]
    page = s["table"][rows].long()
    inside = (idx >= (start // P)[:, None]) & (idx < torch.minimum(have, need)) & (end > start)[:, None]
    shared = inside & (s["refs"][page.clamp(min=0)] > 1)
    who = torch.arange(rows.numel(), device="cuda")[:, None].expand_as(page)
    count = torch.zeros_like(s["refs"]).index_add_(0, page[shared], torch.ones_like(page[shared], dtype=torch.int32))
    last = torch.full_like(s["refs"], -1, dtype=torch.int64).scatter_reduce_(0, page[shared], who[shared], "amax")
    p0 = page.clamp(min=0)
    copy = shared & ~((count[p0] == s["refs"][p0]) & (last[p0] == who))
    add = (idx >= have) & (idx < need)
    n_copy, n_add = copy.sum(1), add.sum(1)
    base = (n_copy + n_add).cumsum(0) - (n_copy + n_add)
    rank = torch.where(copy, base[:, None] + copy.cumsum(1) - 1, base[:, None] + n_copy[:, None] + add.cumsum(1) - 1)
    new = copy | add
    fresh = s["free_list"][(s["free_count"].long() - 1 - rank[new])]
    src, dst = page[copy], s["free_list"][(s["free_count"].long() - 1 - rank[copy])].long()
    s["refs"].index_add_(0, src, torch.full_like(src, -1, dtype=torch.int32))
    s["refs"][fresh.long()] = 1
    t = s["table"][rows]
    t[new] = fresh
    s["table"][rows] = t
    s["row_pages"][rows] = torch.maximum(have, need)[:, 0].to(torch.int32)
    s["free_count"] -= int(new.sum())
    _move(s, src, dst)


def _move(s: dict, src, dst):
    for pool in s["pools"]:
        pool[dst] = pool[src]


def _compact(s: dict):
    """The pages in use moved to the lowest numbers: the k-th page beyond them to the k-th hole."""
    used = s["refs"] > 0
    n = int(used.sum())
    here = torch.arange(used.numel(), device="cuda")
    src, dst = here[used & (here >= n)], here[~used & (here < n)]
    to = here.clone()
    to[src] = dst
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()].to(torch.int32), s["table"]))
    s["refs"][dst] = s["refs"][src]
    s["refs"][src] = 0
    left = used.numel() - n
    s["free_list"][:left] = here[n:].flip(0).to(torch.int32)
    s["free_count"].fill_(left)
    _move(s, src, dst)


def _run_pages(s: dict):
    case, P = s["case"], s["case"]["page"]
    names = ("table", "row_pages", "refs", "free_list", "free_count")
    if case["what"] == "fork":
        if own:
            c = _ctx()
            c.pages_free(s["pt"], s["dst"])
            c.pages_fork(s["pt"], s["src"], s["dst"])
            c.pages_reserve(s["pt"], s["dst"], s["start"], add=case["add"])
            if case["states"]:
                c.rows_copy(s["state_rows"], s["src"], s["dst"])
        else:
            _free(s, s["dst"], P)
            src, dst = s["src"].long(), s["dst"].long()
            s["table"][dst] = s["table"][src]
            s["row_pages"][dst] = s["row_pages"][src]
            page = s["table"][dst][s["table"][dst] >= 0].long()
            s["refs"].index_add_(0, page, torch.ones_like(page, dtype=torch.int32))
            _reserve(s, s["dst"], s["start"], s["start"] + case["add"], P)
            for x in s["states"]:
                x[dst] = x[src]
        return {**{n: s[n] for n in names}, "pools": s["pools"], "states": s["states"]}
    if own:
        c = _ctx()
        c.pages_free(s["pt"], s["rows_a"])
        c.pages_compact(s["pt"])
        c.pages_reserve(s["pt"], s["rows_a"], torch.zeros_like(s["len_a"]), end=s["len_a"])
        c.pages_free(s["pt"], s["rows_b"])
        c.pages_compact(s["pt"])
        c.pages_reserve(s["pt"], s["rows_b"], torch.zeros_like(s["len_b"]), end=s["len_b"])
    else:
        _free(s, s["rows_a"], P)
        _compact(s)
        _reserve(s, s["rows_a"], torch.zeros_like(s["len_a"]), s["len_a"], P)
        _free(s, s["rows_b"], P)
        _compact(s)
        _reserve(s, s["rows_b"], torch.zeros_like(s["len_b"]), s["len_b"], P)
    return {**{n: s[n] for n in names}, "pools": s["pools"]}


# ---------------------------------------------------------------------------
# what the measurement calls
# ---------------------------------------------------------------------------
_PREPARE = {"rope": _prepare_rope, "write": _prepare_cache, "attn": _prepare_cache, "pages": _prepare_pages}


def prepare(case: dict, seed: int) -> dict:
    return dict(_PREPARE[case["kind"]](case, seed), case=case)


def run(s: dict):
    return {"rope": _run_rope, "write": _run_write, "attn": _run_attn, "pages": _run_pages}[s["case"]["kind"]](s)


def exact(case: dict, seed: int):
    if case["kind"] == "pages":        # numbers of pages, and pages moved as they are: nothing is computed
        return None
    s = prepare(case, seed)
    return {"rope": _exact_rope, "write": _exact_write, "attn": _exact_attn}[case["kind"]](case, s)


def work(case: dict) -> dict:
    kind, B, N, Hq, Hkv = (case.get(n, 0) for n in ("kind", "B", "N", "Hq", "Hkv"))
    if kind == "rope":
        n = B * N * (Hq + Hkv) * case["dh"]
        return {"bytes": float(2 * n * (4 if case["dtype"] == "f32" else 2)), "flops": float(8 * n)}
    if kind == "write":    # read in bf16, written in 4.5 bits; entries moved; read in 4.5 bits, written in bf16
        new, moved = B * N * Hkv * 2, 0 if case["shape"] == "prompt" else B * Hkv * 2 / _P_STOP
        back = new if case["shape"] == "prompt" else B * min(N, _DEEPEST) * Hkv * 2
        return {"bytes": float((new + back) * (256 + 72) + 2 * moved * 72), "flops": float(8 * new * _DH)}
    if kind == "attn":
        keys = case["ctx"] * (1 + 0.75 * (B - 1)) + B * N      # half to full length, one sequence at full length
        return {"bytes": float(keys * Hkv * 144 + B * N * Hq * (2 * 256 + 4)), "flops": float(4 * _DH * keys * N * Hq)}
    page = case["layers"] * case["Hkv"] * 2 * case["page"] * 72
    if case["what"] == "fork":             # one page a continuation copied, recurrent states copied
        return {"bytes": float(2 * case["R"] * case["ways"] * (page + case["states"] * case["Hv"] * _DH * _DH * 4)), "flops": 0.0}
    held = 0.75 * case["R"] * case["ctx"] / case["page"]      # twice, half of them are moved
    return {"bytes": float(2 * page * held), "flops": 0.0}
