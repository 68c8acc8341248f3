"""The operators of a paged key/value cache that grows on the device, each in its plain form and as the library's call:

  plan   lengths of the environments -> new pages in the page table, and row, position and cache slot of every new token
  rope   the queries' and keys' norms per head and their rotation; keys and values into their cache slots
  back   the gradient of those norms and that rotation, for training
  attn   attention of one new token of every environment over its cached pages

Sizes come from the presets of paper_2505_18719_amd/inputs.py (tiny, mid, the OpenVLA-7B decoder shape, 256 visual rows and
a short prompt) and are generic where those end: grouped heads, long histories, half-precision caches.  The cache's pages
are the library's: 16 tokens, keys [page][head][slot][feature], values [page][head][feature][slot]."""
import math

import numpy as np
import torch

DEV = "cuda"
PAGE = 16
EPS = 1e-6
own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
MOST_KEYS = 1 << 18       # tokens of one pass of a plan, and keys of one environment
MOST_BYTES = 1 << 30      # of a pass of the others
MOST_PADDED = 1 << 29     # elements of the keys, every environment padded to the longest (the plain attention holds them)


def listed():
    rope = {"kind": "rope", "least": 1, "pad": 0, "layout": "half", "scaling": "none", "norm": True, "dtype": "bf16"}
    back = {"kind": "back", "layout": "half", "scaling": "none", "norm": True, "dtype": "bf16"}
    attn = {"kind": "attn", "dtype": "bf16"}
    return [
        # a serving step of 64 environments, one new token each: once per step, before every layer's work
        {"name": "plan_decode_b64", "kind": "plan", "envs": 64, "new": 1, "ctx": 4096, "spread": "equal"},
        # 256 observations with their prompts admitted at once
        {"name": "plan_prefill_b256", "kind": "plan", "envs": 256, "new": 1024, "ctx": 0, "spread": "uniform"},
        # one robot, one new token: the 7B decoder's heads, where a launch's latency counts
        {**rope, "name": "rope_b1", "envs": 1, "new": 1, "ctx": 300, "heads": 32, "kv_heads": 32, "hd": 128, "rot": 128},
        # a decode step of a captured batch of 128 of which 5 rows are padding; grouped heads, far positions
        {**rope, "name": "rope_decode_b123", "envs": 123, "new": 1, "ctx": 120000, "heads": 32, "kv_heads": 8, "hd": 128,
         "rot": 128, "pad": 5, "scaling": "bands"},
        # the prefill of 64 observations and prompts (16 to 48 ids) with grouped heads
        {**rope, "name": "rope_prefill_b64", "envs": 64, "least": 272, "new": 304, "ctx": 0, "heads": 32, "kv_heads": 8,
         "hd": 128, "rot": 128},
        # half precision, part of the head rotated in interleaved pairs, no norms, prompts added to a cached history
        {**rope, "name": "rope_append_f16", "envs": 37, "new": 129, "ctx": 999, "heads": 16, "kv_heads": 16, "hd": 64,
         "rot": 32, "layout": "interleaved", "norm": False, "dtype": "f16"},
        # training: the tiny preset's rows, and a minibatch of 64 observations, prompts and actions
        {**back, "name": "back_tiny", "rows": 4 * 279, "heads": 4, "kv_heads": 4, "hd": 64, "rot": 64},
        {**back, "name": "back_b64", "rows": 64 * 295, "heads": 32, "kv_heads": 8, "hd": 128, "rot": 128},
        # one robot's step of the 7B decoder: observation, prompt and the first tokens
        {**attn, "name": "attn_b1", "envs": 1, "len": 278, "spread": "equal", "heads": 32, "kv_heads": 32, "hd": 128},
        # serving: 64 environments with histories of up to 8192 tokens
        {**attn, "name": "attn_b64_ragged", "envs": 64, "len": 8192, "spread": "uniform", "heads": 32, "kv_heads": 8,
         "hd": 128},
        # two long recordings, groups of seven, half precision
        {**attn, "name": "attn_long_f16", "envs": 2, "len": 131072, "spread": "equal", "heads": 28, "kv_heads": 4,
         "hd": 128, "dtype": "f16"},
        # wide heads that all share one key head; one environment is far longer than the others
        {**attn, "name": "attn_b24_hd256", "envs": 24, "len": 6000, "spread": "skew", "heads": 8, "kv_heads": 1, "hd": 256},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _heads(rng):
    hd = rng.choice([64, 128, 128, 256])
    kv = rng.choice([1, 2, 3, 4, 8, 16, 32]) if hd < 256 else rng.choice([1, 2, 4])
    group = rng.choice([g for g in (1, 1, 2, 4, 5, 7, 8, 12, 16, 24, 32) if g * kv <= 64])
    return {"heads": kv * group, "kv_heads": kv, "hd": hd, "dtype": rng.choice(["bf16", "bf16", "f16"])}


def _rotation(rng, hd):
    return {"rot": rng.choice([hd, hd, hd, hd // 2, hd // 4, 48, 0]), "layout": rng.choice(["half", "interleaved"]),
            "scaling": rng.choice(["none", "linear", "bands"]), "norm": rng.random() < 0.7}


def _draw(rng):
    kind = rng.choice(["plan", "rope", "rope", "back", "back", "attn", "attn", "attn"])
    c = {"kind": kind}
    if kind == "plan":
        c["envs"] = _log_int(rng, 1, 2000)
        c["new"] = rng.choice([1, _log_int(rng, 1, MOST_KEYS // c["envs"])])
        c["ctx"] = rng.choice([0, _log_int(rng, 1, 65536)])
        c["spread"] = rng.choice(["equal", "uniform"])
        return c
    c.update(_heads(rng))
    if kind == "attn":
        c["envs"] = _log_int(rng, 1, 300)
        c["len"] = _log_int(rng, 1, MOST_KEYS)
        c["spread"] = rng.choice(["equal", "uniform", "uniform", "skew"])
        return c
    c.update(_rotation(rng, c["hd"]))
    if kind == "back":
        c["rows"] = _log_int(rng, 1, 40000)
        return c
    c["envs"] = _log_int(rng, 1, 300)
    c["least"], c["new"] = 1, rng.choice([1, _log_int(rng, 1, 2000)])
    c["ctx"] = rng.choice([0, _log_int(rng, 1, 1000000)])
    c["pad"] = rng.choice([0, 0, 1, 13])
    return c


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        c = _draw(rng)
        if work(c)["bytes"] > min(most, MOST_BYTES):
            continue
        if c["kind"] == "attn" and c["envs"] * c["len"] * c["kv_heads"] * c["hd"] > MOST_PADDED:
            continue
        return c


# ------------------------------------------------------------------ the sizes
def work(case):
    """Bytes of each input read once and each output written once; the flops of the sums and products."""
    c = case
    if c["kind"] == "plan":
        n, rows = c["envs"], int(_sizes(c, c["envs"], 1, c["new"], c["spread"]).sum())
        return {"bytes": 16 * n + 12 * rows + 8 * rows / PAGE, "flops": 4 * rows}
    hd, H, K = c["hd"], c["heads"], c["kv_heads"]
    if c["kind"] == "attn":
        keys = int(_sizes(c, c["envs"], 1, c["len"], c["spread"]).sum())
        return {"bytes": 4 * keys * K * hd + 4 * c["envs"] * H * hd + 4 * keys / PAGE, "flops": 4 * keys * H * hd}
    if c["kind"] == "rope":
        rows = int(_sizes(c, c["envs"], c["least"], c["new"]).sum())
        return {"bytes": rows * (4 * (H + 2 * K) * hd + 8), "flops": rows * (H + K) * (4 * hd + 6 * c["rot"] / 2)}
    return {"bytes": c["rows"] * (6 * (H + K) * hd + 4), "flops": c["rows"] * (H + K) * (12 * hd + 6 * c["rot"] / 2)}


# ------------------------------------------------------------------ the inputs
def _rand(g, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(dtype)


def _freqs(c):
    """Radians per position of each pair, in 64 bits: base 10000; "linear" stretches the positions 4-fold, "bands" only the
    pairs that turn less than 4 times over the first 8192 positions, 8-fold below one turn and a blend between."""
    n = c["rot"] // 2
    f = 10000.0 ** (-np.arange(n, dtype=np.float64) / max(n, 1))
    if c["scaling"] == "linear":
        f = f / 4
    if c["scaling"] == "bands":
        t = np.clip((8192 * f / (2 * math.pi) - 1) / 3, 0, 1)
        f = f * (t + (1 - t) / 8)
    return f


def _i32(x):
    return torch.from_numpy(np.asarray(x, dtype=np.int32)).to(DEV)


def _sizes(c, n, lo, hi, spread="uniform"):
    """n whole numbers that belong to the case, so that its shapes do: all hi, spread over lo .. hi, or one hi among ones of
    up to a sixteenth of it.  Which environment has which is the seed's."""
    if spread == "equal":
        return np.full(n, hi, dtype=np.int64)
    rng = np.random.default_rng([n, lo, hi, len(spread), 17])
    if spread == "skew":
        lo, hi, longest = 1, hi // 16 + 1, hi
    out = rng.integers(lo, hi + 1, n)
    if spread == "skew":
        out[0] = longest
    return out


def _pages(tokens):
    return -(-tokens // PAGE)


def prepare(case, seed):
    rng = np.random.default_rng([seed, 71])
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 5)
    s = {"case": case, **globals()["_prepare_" + case["kind"]](case, rng, g)}
    if own:
        from paper_2505_18719_amd import vla
        s["vla"] = vla
        if case["kind"] == "attn":
            s["ws"] = vla.paged_attention_workspace(s["q"], s["k_pages"], s["page_table"])
        if case["kind"] == "back":
            s["ws"] = vla.qk_norm_rope_workspace(s["q"])
    return s


def _prepare_plan(c, rng, g):
    n = c["envs"]
    cached = rng.permutation(_sizes(c, n, 0, c["ctx"]))
    new = rng.permutation(_sizes(c, n, 1, c["new"], c["spread"]))
    held, width = _pages(cached), int(_pages(cached.max() + new.max())) + 2
    n_pages = int((held + _pages(new)).sum()) + 40
    pages = rng.permutation(n_pages)
    table = np.full((n, width), -1, dtype=np.int32)
    at = 0
    for i in range(n):
        table[i, :held[i]] = pages[at:at + held[i]]
        at += int(held[i])
    return {"cached": _i32(cached), "new": _i32(new), "page_table": _i32(table), "free": _i32(pages[at:]),
            "head": _i32([3]), "n_pages": n_pages, "max_rows": int(new.sum()) + 7}


def _prepare_rope(c, rng, g):
    n, H, K, hd, dt = c["envs"], c["heads"], c["kv_heads"], c["hd"], DTYPES[c["dtype"]]
    cached = rng.permutation(_sizes(c, n, 0, c["ctx"]))
    new = rng.permutation(_sizes(c, n, c["least"], c["new"]))
    first, last = cached // PAGE, (cached + new - 1) // PAGE
    held = last - first + 1  # pages of the pool that this pass touches
    n_pages = int(_pages(new).sum()) + n + 5
    pages = rng.permutation(n_pages)
    pos, slot, at = [], [], 0
    for i in range(n):
        p = cached[i] + np.arange(new[i])
        pos.append(p)
        slot.append(pages[at + p // PAGE - first[i]] * PAGE + p % PAGE)
        at += int(held[i])
    pos = np.concatenate(pos + [np.zeros(c["pad"], dtype=np.int64)])
    slot = np.concatenate(slot + [np.full(c["pad"], -1)])
    rows = len(pos)
    qkv = _rand(g, (rows, (H + 2 * K) * hd), dt, 2.0)
    q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([H * hd, K * hd, K * hd], 1))
    gains = (1 + _rand(g, (2, hd), torch.float32, 0.2)).to(dt) if c["norm"] else (None, None)
    return {"q": q, "k": k, "v": v, "q_gain": gains[0], "k_gain": gains[1], "pos": _i32(pos), "slot": _i32(slot),
            "freqs": torch.from_numpy(_freqs(c)).to(DEV), "k_pages": _rand(g, (n_pages, K, PAGE, hd), dt),
            "v_pages": _rand(g, (n_pages, K, hd, PAGE), dt), "out": torch.zeros((rows, H, hd), dtype=dt, device=DEV)}


def _prepare_back(c, rng, g):
    rows, H, K, hd, dt = c["rows"], c["heads"], c["kv_heads"], c["hd"], DTYPES[c["dtype"]]
    qk = _rand(g, (rows, (H + K) * hd), dt, 2.0)
    q, k = (t.unflatten(1, (-1, hd)) for t in qk.split([H * hd, K * hd], 1))
    gains = (1 + _rand(g, (2, hd), torch.float32, 0.2)).to(dt) if c["norm"] else (None, None)
    return {"q": q, "k": k, "dq": _rand(g, (rows, H, hd), dt, 0.1), "dk": _rand(g, (rows, K, hd), dt, 0.1),
            "q_gain": gains[0], "k_gain": gains[1], "pos": _i32(np.arange(rows) % 2048),
            "freqs": torch.from_numpy(_freqs(c)).to(DEV)}


def _prepare_attn(c, rng, g):
    n, H, K, hd, dt = c["envs"], c["heads"], c["kv_heads"], c["hd"], DTYPES[c["dtype"]]
    lens = rng.permutation(_sizes(c, n, 1, c["len"], c["spread"]))
    held = _pages(lens)
    n_pages = int(held.sum()) + 3
    pages = rng.permutation(n_pages)
    table = np.full((n, int(held.max()) + 1), -1, dtype=np.int32)  # entries past a sequence name no page
    at = 0
    for i in range(n):
        table[i, :held[i]] = pages[at:at + held[i]]
        at += int(held[i])
    k_pages, v_pages = _rand(g, (n_pages, K, PAGE, hd), dt), _rand(g, (n_pages, K, hd, PAGE), dt)
    last = torch.from_numpy(table[np.arange(n), held - 1].astype(np.int64)).to(DEV)
    fill = torch.from_numpy((lens - 1) % PAGE + 1).to(DEV)
    dead = torch.arange(PAGE, device=DEV)[None] >= fill[:, None]  # slots of the last page that hold no token yet
    k_pages[last] = k_pages[last].masked_fill(dead[:, None, :, None], float("nan"))
    v_pages[last] = v_pages[last].masked_fill(dead[:, None, None, :], float("nan"))
    return {"q": _rand(g, (n, H, hd), dt, 2.0), "k_pages": k_pages, "v_pages": v_pages, "page_table": _i32(table),
            "lens": _i32(lens), "scale": hd ** -0.5, "out": torch.empty((n, H, hd), dtype=dt, device=DEV)}


# ------------------------------------------------------------------ one pass
def run(s):
    c, kind = s["case"], s["case"]["kind"]
    if not own:
        return globals()["_plain_" + kind](s)
    vla = s["vla"]
    if kind == "plan":
        o = vla.kv_plan(s["cached"], s["new"], s["page_table"], s["free"], s["n_pages"], s["max_rows"], free_head=s["head"])
        return {**o, "page_table": s["page_table"]}
    if kind == "rope":
        vla.qk_norm_rope(s["q"], s["k"], s["pos"], s["freqs"], s["q_gain"], s["k_gain"], EPS, c["layout"], v=s["v"],
                         k_pages=s["k_pages"], v_pages=s["v_pages"], row_slot=s["slot"], q_out=s["out"])
        return {"q": s["out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if kind == "back":
        dq, dk, dqg, dkg = vla.qk_norm_rope_backward(s["q"], s["k"], s["dq"], s["dk"], s["pos"], s["freqs"], s["q_gain"],
                                                     s["k_gain"], EPS, c["layout"], workspace=s["ws"])
        return {"dq": dq, "dk": dk, **({"dq_gain": dqg, "dk_gain": dkg} if c["norm"] else {})}
    return vla.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["lens"], s["scale"], out=s["out"],
                               workspace=s["ws"])


# ------------------------------------------------------------------ the plain forms
def _plain_plan(s):
    cached, new, table, free = s["cached"].long(), s["new"].long(), s["page_table"], s["free"]
    n, width = table.shape
    rows = s["max_rows"]
    head = s["head"].long()
    end = new.cumsum(0)
    held, want = (cached + PAGE - 1) // PAGE, (cached + new + PAGE - 1) // PAGE
    fits = (want <= width) & (end <= rows)
    need = torch.where(fits, want - held, 0)
    taken = need.cumsum(0)
    ok = fits & ((need == 0) | (head + taken <= free.numel()))
    need = torch.where(ok, need, 0)
    taken = need.cumsum(0)
    col = torch.arange(width, device=DEV)[None]
    fresh = (col >= held[:, None]) & (col < (held + need)[:, None])
    at = head + (taken - need)[:, None] + col - held[:, None]
    table.copy_(torch.where(fresh, free[at.clamp(0, free.numel() - 1)], table))
    row = torch.arange(rows, device=DEV)
    env = torch.searchsorted(end, row, right=True)
    live = env < n
    env = env.clamp(max=n - 1)
    pos = cached[env] + row - (end - new)[env]
    page = table[env, (pos // PAGE).clamp(max=width - 1)].long()
    good = live & ok[env] & (page >= 0) & (page < s["n_pages"])
    return {"lens": torch.where(ok, cached + new, cached).int(), "row_start": torch.cat([end.new_zeros(1), end]).int(),
            "row_pos": torch.where(live, pos, 0).int(), "row_env": torch.where(live, env, -1).int(),
            "row_slot": torch.where(good, page * PAGE + pos % PAGE, -1).int(),
            "stats": torch.stack([head[0] + taken[-1], end[-1], (~ok).sum()]).int(), "page_table": table}


def _cos_sin(s, dtype):
    t = s["pos"].double()[:, None, None] * s["freqs"]
    return t.cos().to(dtype), t.sin().to(dtype)


def _pairs(x, rot, layout):
    if layout == "half":
        return x[..., :rot // 2], x[..., rot // 2:rot]
    return x[..., 0:rot:2], x[..., 1:rot:2]


def _turn(x, cos, sin, rot, layout):
    a, b = _pairs(x, rot, layout)
    y = x.clone()
    ya, yb = _pairs(y, rot, layout)
    ya.copy_(a * cos - b * sin)
    yb.copy_(b * cos + a * sin)
    return y


def _norm_turn(s, x, gain, cos, sin):
    c = s["case"]
    x = x.to(cos.dtype)
    if gain is not None:
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * gain.to(cos.dtype)
    return _turn(x, cos, sin, c["rot"], c["layout"])


def _plain_rope(s):
    dt = s["out"].dtype
    cos, sin = _cos_sin(s, torch.float32)
    live = s["slot"] >= 0
    slot = s["slot"][live].long()
    page, at = slot // PAGE, slot % PAGE
    q = _norm_turn(s, s["q"], s["q_gain"], cos, sin).to(dt)
    s["out"].copy_(torch.where(live[:, None, None], q, s["out"]))
    s["k_pages"][page, :, at] = _norm_turn(s, s["k"], s["k_gain"], cos, sin).to(dt)[live]
    s["v_pages"][page, :, :, at] = s["v"][live]
    return {"q": s["out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_back(s):
    c = s["case"]
    cos, sin = _cos_sin(s, torch.float32)
    out = {}
    for name in ("q", "k"):
        x, gain = s[name].float(), s[name + "_gain"]
        dy = _turn(s["d" + name].float(), cos, -sin, c["rot"], c["layout"])
        if gain is not None:
            r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
            h = x * r
            out["d" + name + "_gain"] = (dy * h).sum((0, 1), dtype=torch.float64).float()
            dy = dy * gain.float()
            dy = r * (dy - h * (dy * h).mean(-1, keepdim=True))
        out["d" + name] = dy.to(s[name].dtype)
    return {k: out[k] for k in ("dq", "dk", "dq_gain", "dk_gain") if k in out}


def _plain_attn(s):
    c, q, table, lens = s["case"], s["q"], s["page_table"], s["lens"]
    n, H, hd = q.shape
    K, L = c["kv_heads"], table.shape[1] * PAGE
    idx = table.clamp(min=0).long()
    keys = s["k_pages"][idx].float().permute(0, 2, 1, 3, 4).reshape(n * K, L, hd)
    scores = torch.bmm(keys, q.float().reshape(n * K, H // K, hd).transpose(1, 2).contiguous() * s["scale"])
    del keys
    dead = torch.arange(L, device=DEV)[None] >= lens[:, None]
    dead_k = dead[:, None].expand(n, K, L).reshape(n * K, L)
    p = (scores.masked_fill(dead_k[:, :, None], -math.inf)).softmax(1)
    vals = s["v_pages"][idx].float().permute(0, 2, 3, 1, 4).reshape(n * K, hd, L).masked_fill(dead_k[:, None], 0.0)
    o = torch.bmm(vals, p).transpose(1, 2).reshape(n, H, hd).to(q.dtype)
    return torch.where((lens > 0)[:, None, None], o, 0)


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return globals()["_exact_" + case["kind"]](s)


def _exact_plan(s):
    """One environment after the other, one token after the other."""
    cached, new, free = s["cached"].tolist(), s["new"].tolist(), s["free"].tolist()
    table = s["page_table"].cpu().numpy().copy()
    rows = s["max_rows"]
    at = int(s["head"])
    pos, env, slot = np.zeros(rows, np.int32), np.full(rows, -1, np.int32), np.full(rows, -1, np.int32)
    lens, start, refused = list(cached), [0], 0
    for i, (c, w) in enumerate(zip(cached, new)):
        r0 = start[-1]
        start.append(r0 + w)
        p = np.arange(c, c + w)
        pos[r0:r0 + w], env[r0:r0 + w] = p, i
        have, want = _pages(c), _pages(c + w)
        if at + want - have > len(free):
            refused += 1
            continue
        table[i, have:want] = free[at:at + want - have]
        at += want - have
        lens[i] = c + w
        slot[r0:r0 + w] = table[i, p // PAGE] * PAGE + p % PAGE
    return {"lens": _i32(lens), "row_start": _i32(start), "row_pos": _i32(pos), "row_env": _i32(env), "row_slot": _i32(slot),
            "stats": _i32([at, start[-1], refused]), "page_table": _i32(table)}


def _rotation64(s):
    """[rows, 1, hd / 2 or fewer] complex factors e^(i t)."""
    return torch.exp(1j * (s["pos"].double()[:, None, None] * s["freqs"]))


def _turn64(x, factor, rot, layout):
    head, rest = x[..., :rot], x[..., rot:]
    z = head.unflatten(-1, (2, -1)).transpose(-1, -2) if layout == "half" else head.unflatten(-1, (-1, 2))
    w = torch.view_as_real(torch.view_as_complex(z.contiguous()) * factor)
    w = w.transpose(-1, -2) if layout == "half" else w
    return torch.cat([w.flatten(-2), rest], -1)


def _exact_rope(s):
    c, z = s["case"], _rotation64(s)
    new = {}
    for name in ("q", "k"):
        x, gain = s[name].double(), s[name + "_gain"]
        if gain is not None:
            x = gain.double() * x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["hd"] + EPS)
        new[name] = _turn64(x, z, c["rot"], c["layout"])
    slots = s["slot"].tolist()
    rows = [r for r, t in enumerate(slots) if t >= 0]
    t = torch.tensor([slots[r] for r in rows], device=DEV)
    out = s["out"].double()
    out[rows] = new["q"][rows]
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    K, hd = c["kv_heads"], c["hd"]
    flat = kp.transpose(1, 2).reshape(-1, K, hd)
    flat[t] = new["k"][rows]
    kp = flat.unflatten(0, (-1, PAGE)).transpose(1, 2).contiguous()
    flat = vp.permute(0, 3, 1, 2).reshape(-1, K, hd)
    flat[t] = s["v"].double()[rows]
    vp = flat.unflatten(0, (-1, PAGE)).permute(0, 2, 3, 1).contiguous()
    return {"q": out, "k_pages": kp, "v_pages": vp}


def _exact_back(s):
    """The gradient of sum(out * dout) by automatic differentiation of the definition."""
    c, z = s["case"], _rotation64(s)
    out = {}
    for name in ("q", "k"):
        x = s[name].double().requires_grad_()
        gain = None if s[name + "_gain"] is None else s[name + "_gain"].double().requires_grad_()
        y = x
        if gain is not None:
            y = gain * x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["hd"] + EPS)
        loss = (_turn64(y, z, c["rot"], c["layout"]) * s["d" + name].double()).sum()
        grads = torch.autograd.grad(loss, [x] + ([] if gain is None else [gain]))
        out["d" + name] = grads[0]
        if gain is not None:
            out["d" + name + "_gain"] = grads[1]
    return {k: out[k] for k in ("dq", "dk", "dq_gain", "dk_gain") if k in out}


def _exact_attn(s):
    """Per environment and key head: exp of the scores over their sum, weighting the values."""
    c, lens, table = s["case"], s["lens"].tolist(), s["page_table"].long()
    K, hd = c["kv_heads"], c["hd"]
    G = c["heads"] // K
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for i, n in enumerate(lens):
        if n == 0:
            continue
        pages = table[i, :(n + PAGE - 1) // PAGE]
        for h in range(K):
            k = s["k_pages"][pages, h].reshape(-1, hd)[:n].double()
            v = s["v_pages"][pages, h].transpose(1, 2).reshape(-1, hd)[:n].double()
            for j in range(h * G, (h + 1) * G):
                t = (k * s["q"][i, j].double()).sum(1) * s["scale"]
                w = torch.exp(t - t.max())
                out[i, j] = (w[:, None] * v).sum(0) / w.sum()
    return out
