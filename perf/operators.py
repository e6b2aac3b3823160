"""Workloads of the transformer operators: rotary positions, appending to a paged key-value cache, attention of one new
token over that cache, and the root-mean-square norm with residual addition, 8-bit output and gradient.

`listed()` and `draw()` give cases, `prepare()` the data a serving or training loop has in hand, `run()` one pass through
an operator: in plain torch operations where `own` is false, through the package's public entry points where it is true.
`exact()` evaluates the definition in 64 bits, `work()` counts the bytes and operations a pass cannot do without.
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # One conversation, one thousand tokens into it: a decode step's attention where only latency counts.
        dict(name="attend_one", op="attend", batch=1, heads=32, kv_heads=8, dim=128, page=16, longest=1013, shortest=1013, empty=0, dtype="bf16", head_major=True),
        # A handful of long documents of uneven length: the cache has to be split along its length.
        dict(name="attend_long", op="attend", batch=4, heads=32, kv_heads=8, dim=128, page=64, longest=32768, shortest=7001, empty=0, dtype="bf16", head_major=True),
        # A full serving batch, padded with rows that hold no sequence, lengths spread from a few tokens to thousands.
        dict(name="attend_batch", op="attend", batch=64, heads=32, kv_heads=8, dim=128, page=16, longest=4096, shortest=17, empty=3, dtype="bf16", head_major=False),
        # Every query head with keys of its own, 32-bit values, narrow heads.
        dict(name="attend_f32", op="attend", batch=16, heads=16, kv_heads=16, dim=64, page=32, longest=2048, shortest=255, empty=0, dtype="f32", head_major=True),
        # The newest token of one sequence, far into a long context.
        dict(name="rotary_one", op="rotary", tokens=1, heads=32, dim=128, rotated=128, interleaved=False, inverse=False, scaling="none", dtype="bf16", far=131072),
        # A prompt in 32 bits: interleaved pairs, half of an odd-sized head rotated.
        dict(name="rotary_prompt_f32", op="rotary", tokens=2048, heads=16, dim=80, rotated=40, interleaved=True, inverse=False, scaling="linear", dtype="f32", far=16384),
        # The gradient through the rotation for a long training sequence, frequencies stretched for long contexts.
        dict(name="rotary_gradient", op="rotary", tokens=8192, heads=32, dim=128, rotated=128, interleaved=False, inverse=True, scaling="parts", dtype="bf16", far=8192),
        # A decode step of a batch: one key and value per sequence, some rows padding.
        dict(name="append_step", op="append", tokens=64, heads=32, kv_heads=8, dim=128, page=16, pages=1024, padding=5, packed=False, dtype="bf16", head_major=True),
        # Several prompts at once, keys and values being slices of one packed projection.
        dict(name="append_prompt", op="append", tokens=8192, heads=32, kv_heads=8, dim=128, page=64, pages=192, padding=100, packed=True, dtype="bf16", head_major=False),
        # The norm of a decode step, its output in 8 bits with one scale per row for the projection that follows.
        dict(name="norm_step", op="norm", rows=16, cols=4096, group=0, eight=True, residual=True, dtype="bf16"),
        # The norm of a prompt, 8 bits with a scale for every 128 values.
        dict(name="norm_prompt", op="norm", rows=8192, cols=4096, group=128, eight=True, residual=True, dtype="bf16"),
        # The gradient of the norm over a training batch, with the gradient that reaches the residual stream directly.
        dict(name="norm_gradient", op="norm_gradient", rows=16384, cols=1024, residual=True, dtype="bf16"),
    ]


def _log_range(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "rotary", "append", "norm", "norm_gradient"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    size = 2 if dtype == "bf16" else 4
    if op == "attend":
        dim = rng.choice([64, 128, 128, 80, 96, 256])
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.choice([1, 2, 4, 5, 8, 16])
        batch = _log_range(rng, 1, 96)
        most = max(2, min(32768, (300 << 20) // (batch * kv_heads * dim * 2 * size)))
        longest = _log_range(rng, 1, most)
        return dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, dim=dim, page=rng.choice([8, 16, 32, 48, 64]), longest=longest,
                    shortest=rng.randint(1, longest), empty=rng.choice([0, 0, 1]) if batch > 2 else 0, dtype=dtype, head_major=rng.random() < 0.5)
    if op == "rotary":
        dim = rng.choice([64, 80, 96, 128, 256])
        heads = rng.randint(1, 40)
        tokens = _log_range(rng, 1, (32 << 20) // (heads * dim * size) + 1)
        return dict(op=op, tokens=tokens, heads=heads, dim=dim, rotated=rng.choice([dim, dim // 2, 32]), interleaved=rng.random() < 0.5,
                    inverse=rng.random() < 0.4, scaling=rng.choice(["none", "linear", "parts"]), dtype=dtype, far=_log_range(rng, tokens + 1, 1 << 20))
    if op == "append":
        dim = rng.choice([64, 80, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        tokens = _log_range(rng, 1, (16 << 20) // (kv_heads * dim * 2 * size) + 1)
        page = rng.choice([8, 16, 32, 48, 64])
        return dict(op=op, tokens=tokens, heads=kv_heads * rng.choice([1, 4]), kv_heads=kv_heads, dim=dim, page=page, pages=tokens // page + rng.randint(2, 40),
                    padding=rng.randint(0, tokens // 8), packed=rng.random() < 0.5, dtype=dtype, head_major=rng.random() < 0.5)
    cols = rng.choice([rng.randint(64, 1000), 8 * rng.randint(16, 1024), 1024, 2048, 4096, 8192])
    rows = _log_range(rng, 1, (32 << 20) // (cols * size) + 1)
    if op == "norm":
        eight = rng.random() < 0.6
        return dict(op=op, rows=rows, cols=cols, group=rng.choice([0, 32, 64, 128]) if eight else 0, eight=eight, residual=rng.random() < 0.7, dtype=dtype)
    return dict(op=op, rows=rows, cols=cols, residual=rng.random() < 0.5, dtype=dtype)


def _lengths(case):
    """Tokens each sequence of an attention case holds: spread from the shortest to the longest, in no order; the last rows are empty."""
    held = case["batch"] - case["empty"]
    low, high = case["shortest"], case["longest"]
    n = [high if held == 1 else low + (high - low) * i // (held - 1) for i in range(held)]
    random.Random(7 * held + high).shuffle(n)
    return n + [0] * case["empty"]


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


SCALING = {  # how the frequencies are changed for contexts longer than the training one
    "none": dict(base=10000.0, kind="none"),
    "linear": dict(base=10000.0, kind="linear", factor=4.0),
    "parts": dict(base=500000.0, kind="parts", factor=8.0, original_length=8192, low=1.0, high=4.0),
}


def _frequencies(rotated, base, kind, factor=1.0, original_length=0, low=1.0, high=4.0):
    """Radians per position of each pair: base^(-2i/rotated), divided by the factor ("linear") or only as far as a pair makes few turns in the original length ("parts")."""
    f = torch.pow(torch.tensor(base, dtype=torch.float64), -torch.arange(0, rotated, 2, dtype=torch.float64) / rotated)
    if kind == "linear":
        f = f / factor
    elif kind == "parts":
        keep = ((original_length * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _type(case)

    def normal(*shape, std=1.0):
        x = torch.empty(shape, device="cuda", dtype=t).normal_(0.0, std, generator=g)
        return x

    op = case["op"]
    s = {"case": dict(case)}
    if op == "attend":
        n = _lengths(case)
        page, kv_heads, dim = case["page"], case["kv_heads"], case["dim"]
        per = [-(-x // page) for x in n]
        pages = sum(per) + 3
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        width = max(per) + 1
        first = torch.tensor([sum(per[:i]) for i in range(len(per))], device="cuda")
        at = first[:, None] + torch.arange(width, device="cuda")[None, :]
        used = torch.arange(width, device="cuda")[None, :] < torch.tensor(per, device="cuda")[:, None]
        s["page_table"] = torch.where(used, order[at.clamp(max=pages - 1)], -1).to(torch.int32)  # entries behind a sequence's last page name none
        s["lengths"] = torch.tensor(n, device="cuda", dtype=torch.int32)
        shape = (pages, 2, kv_heads, page, dim) if case["head_major"] else (pages, 2, page, kv_heads, dim)
        s["cache"] = normal(*shape)
        s["q"] = normal(len(n), case["heads"], dim, std=1.5)
        s["out"] = torch.empty_like(s["q"])
    elif op == "rotary":
        s["x"] = normal(case["tokens"], case["heads"], case["dim"])
        start = torch.randint(0, max(1, case["far"] - case["tokens"]), (1,), device="cuda", generator=g)
        s["positions"] = (start + torch.arange(case["tokens"], device="cuda")).to(torch.int32)
        s["frequencies"] = _frequencies(case["rotated"], **SCALING[case["scaling"]]).cuda()
        s["out"] = torch.empty_like(s["x"])
    elif op == "append":
        n, page, pages, heads, kv_heads, dim = (case[k] for k in ("tokens", "page", "pages", "heads", "kv_heads", "dim"))
        shape = (pages, 2, kv_heads, page, dim) if case["head_major"] else (pages, 2, page, kv_heads, dim)
        s["cache"] = normal(*shape)
        slots = torch.randperm(pages * page, device="cuda", generator=g)[:n]
        if n > 256:  # prompts fill pages from front to back
            order = torch.randperm(pages, device="cuda", generator=g)
            slots = (order[:, None] * page + torch.arange(page, device="cuda")[None, :]).reshape(-1)[:n]
        s["slots"] = slots.to(torch.int32)
        if case["padding"]:
            s["slots"][n - case["padding"]:] = -1  # rows behind the last sequence
        s["positions"] = torch.randint(0, 32768, (n,), device="cuda", generator=g, dtype=torch.int32)
        s["frequencies"] = _frequencies(dim, **SCALING["none"]).cuda()
        if case["packed"]:
            s["qkv"] = normal(n, heads + 2 * kv_heads, dim)
        else:
            s["k"], s["v"] = normal(n, kv_heads, dim), normal(n, kv_heads, dim)
    elif op == "norm":
        rows, cols = case["rows"], case["cols"]
        s["x"] = normal(rows, cols)
        if case["residual"]:
            s["residual"] = normal(rows, cols, std=2.0)
        s["gamma"] = 1 + torch.empty(cols, device="cuda").normal_(0.0, 0.1, generator=g)
    else:
        rows, cols = case["rows"], case["cols"]
        s["dy"], s["h"] = normal(rows, cols, std=0.1), normal(rows, cols, std=2.0)
        if case["residual"]:
            s["dsum"] = normal(rows, cols, std=0.1)
        s["gamma"] = 1 + torch.empty(cols, device="cuda").normal_(0.0, 0.1, generator=g)
    return s


EPS = 1e-6


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, positions, frequencies, interleaved, inverse):
    """x [tokens, heads, dim], in 32 bits; angles in 64."""
    angle = positions.double()[:, None] * frequencies[None, :]
    if inverse:
        angle = -angle
    c, s = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    r = 2 * frequencies.numel()
    x = x.float()
    if interleaved:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * c - b * s, a * s + b * c), dim=-1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2: r]
        turned = torch.cat((a * c - b * s, a * s + b * c), dim=-1)
    return torch.cat((turned, x[..., r:]), dim=-1)


def _attend(s):
    case, cache, table, n = s["case"], s["cache"], s["page_table"], s["lengths"]
    kv = cache[table.clamp(min=0).long()]  # [batch, pages, 2, ...]
    kv = kv.permute(0, 2, 3, 1, 4, 5) if case["head_major"] else kv.permute(0, 2, 4, 1, 3, 5)  # [batch, 2, kv heads, pages, page, dim]
    batch, dim = kv.shape[0], kv.shape[-1]
    kv = kv.reshape(batch, 2, case["kv_heads"], -1, dim).float()
    q = s["q"].float().reshape(batch, case["kv_heads"], -1, dim)
    score = torch.matmul(q, kv[:, 0].transpose(-1, -2)) * dim ** -0.5
    there = torch.arange(score.shape[-1], device=score.device)[None, :] < n[:, None]
    score = score.masked_fill(~there[:, None, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    v = kv[:, 1].masked_fill(~there[:, None, :, None], 0.0)
    out = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    s["out"].copy_(out.reshape(s["out"].shape))
    return [s["out"]]


def _append(s):
    case, cache = s["case"], s["cache"]
    kv_heads, heads, page = case["kv_heads"], case["heads"], case["page"]
    k = s["qkv"][:, heads: heads + kv_heads] if case["packed"] else s["k"]
    v = s["qkv"][:, heads + kv_heads:] if case["packed"] else s["v"]
    k = _rotate(k, s["positions"], s["frequencies"], False, False).to(cache.dtype)
    slots = s["slots"].long()
    kept = torch.arange(slots.numel(), device=slots.device)[: slots.numel() - case["padding"]]
    at, off = slots[kept] // page, slots[kept] % page
    if case["head_major"]:
        cache[at, 0, :, off] = k[kept]
        cache[at, 1, :, off] = v[kept]
    else:
        cache[at, 0, off] = k[kept]
        cache[at, 1, off] = v[kept]
    return [cache]


def _norm(s):
    case = s["case"]
    h = s["x"].float() + s["residual"].float() if case["residual"] else s["x"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["gamma"]
    outs = [h.to(s["x"].dtype)] if case["residual"] else []
    if not case["eight"]:
        return [y.to(s["x"].dtype)] + outs
    rows, cols = y.shape
    group = case["group"] or cols
    groups = -(-cols // group)
    if groups * group != cols:
        y = torch.cat((y, y.new_zeros(rows, groups * group - cols)), dim=-1)
    y = y.reshape(rows, groups, group)
    top = y.abs().amax(-1, keepdim=True)
    codes = (y * torch.where(top > 0, E4M3_MAX / top, 0.0)).to(torch.float8_e4m3fn)
    return [codes.reshape(rows, -1)[:, :cols], (top / E4M3_MAX).reshape(rows, groups)] + outs


def _norm_gradient(s):
    dy, h = s["dy"].float(), s["h"].float()
    inverse = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    unit = h * inverse
    d = dy * s["gamma"]
    dx = inverse * (d - unit * (d * unit).mean(-1, keepdim=True))
    if s["case"]["residual"]:
        dx = dx + s["dsum"].float()
    return [dx.to(s["h"].dtype), (dy * unit).sum(0)]


# ------------------------------------------------------------------------------------------------ the package's operators
_shared = {}


def _context():
    """The program's one context on the device."""
    if "context" not in _shared:
        import paper_2102_13267_b200 as lt

        _shared["lt"], _shared["context"] = lt, lt.LazyContext(device=0)
    return _shared["lt"], _shared["context"]


def _program(s):
    """What a program writes once: handles of its buffers, and the step that it records on them every time."""
    lt, ctx = _context()
    case, op = s["case"], s["case"]["op"]
    b, handles = lt.Batch(), []

    def use(x, dtype=None):
        handles.append(ctx.from_torch(x, dtype))
        return b.input()

    if op == "attend":
        q, cache, table, n, out = (use(s[k]) for k in ("q", "cache", "page_table", "lengths", "out"))
        b.paged_attention(q, cache, table, n, scale=case["dim"] ** -0.5, head_major=case["head_major"], out=out)
        results = [s["out"]]
    elif op == "rotary":
        table = torch.from_numpy(lt.rotary_table(case["rotated"], **SCALING[case["scaling"]]).view("int32")).cuda()
        x, positions, f, out = use(s["x"]), use(s["positions"]), use(table, "u32"), use(s["out"])
        b.rotary(x, positions, f, interleaved=case["interleaved"], inverse=case["inverse"], out=out)
        results = [s["out"]]
    elif op == "append":
        table = torch.from_numpy(lt.rotary_table(case["dim"], **SCALING["none"]).view("int32")).cuda()
        cache, slots, positions, f = use(s["cache"]), use(s["slots"]), use(s["positions"]), use(table, "u32")
        if case["packed"]:
            qkv = use(s["qkv"])
            k = b.op("narrow", qkv, dim=1, start=case["heads"], length=case["kv_heads"])
            v = b.op("narrow", qkv, dim=1, start=case["heads"] + case["kv_heads"], length=case["kv_heads"])
        else:
            k, v = use(s["k"]), use(s["v"])
        b.cache_append(cache, k, v, slots, positions, f, head_major=case["head_major"])
        results = [s["cache"]]
    elif op == "norm":
        rows, cols = case["rows"], case["cols"]
        x, gamma = use(s["x"]), use(s["gamma"])
        residual = use(s["residual"]) if case["residual"] else None
        results = []
        if case["eight"]:
            results += [torch.empty(rows, cols, device="cuda", dtype=torch.float8_e4m3fn),
                        torch.empty(rows, -(-cols // case["group"]) if case["group"] else 1, device="cuda")]
        else:
            results.append(torch.empty_like(s["x"]))
        if case["residual"]:
            results.append(torch.empty_like(s["x"]))
        out = [use(r.view(torch.uint8) if r.dtype == torch.float8_e4m3fn else r) for r in results]
        b.rms_norm(x, gamma, residual=residual, eps=EPS, eight_bit=case["eight"], group=case["group"], out=out)
    else:
        dy, h, gamma = use(s["dy"]), use(s["h"]), use(s["gamma"])
        residual = use(s["dsum"]) if case["residual"] else None
        results = [torch.empty_like(s["h"]), torch.empty_like(s["gamma"])]
        b.rms_norm_grad(dy, h, gamma, residual_grad=residual, eps=EPS, out=[use(r) for r in results])
    return ctx, b, handles, results


def run(state):
    if own:
        if "program" not in state:
            state["program"] = _program(state)
        ctx, step, handles, results = state["program"]
        ctx.record(step, handles)
        ctx.barrier()
        return results
    op = state["case"]["op"]
    if op == "attend":
        return _attend(state)
    if op == "rotary":
        case = state["case"]
        state["out"].copy_(_rotate(state["x"], state["positions"], state["frequencies"], case["interleaved"], case["inverse"]))
        return [state["out"]]
    if op == "append":
        return _append(state)
    return _norm(state) if op == "norm" else _norm_gradient(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, size = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "attend":
        n = _lengths(case)
        table = sum(-(-x // case["page"]) for x in n) * 4 + 4 * len(n)
        return {"bytes": sum(n) * case["kv_heads"] * case["dim"] * 2 * size + 2 * len(n) * case["heads"] * case["dim"] * size + table,
                "flops": 4 * sum(n) * case["heads"] * case["dim"]}
    if op == "rotary":
        values = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * values * size + 4 * case["tokens"] + 4 * case["rotated"], "flops": 3 * case["tokens"] * case["heads"] * case["rotated"]}
    if op == "append":
        kept = case["tokens"] - case["padding"]
        return {"bytes": 4 * kept * case["kv_heads"] * case["dim"] * size + 8 * case["tokens"] + 4 * case["dim"], "flops": 3 * kept * case["kv_heads"] * case["dim"]}
    values = case["rows"] * case["cols"]
    if op == "norm":
        groups = -(-case["cols"] // case["group"]) if case["group"] else 1
        written = values + 4 * case["rows"] * groups if case["eight"] else values * size
        return {"bytes": values * size * (3 if case["residual"] else 1) + written + 4 * case["cols"], "flops": 6 * values}
    return {"bytes": values * size * (4 if case["residual"] else 3) + 8 * case["cols"], "flops": 12 * values}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _turned(x, positions, frequencies, interleaved, inverse):
    z = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), (-1.0 if inverse else 1.0) * positions.double()[:, None, None] * frequencies)
    r = 2 * frequencies.numel()
    head = x[..., :r].double()
    pairs = head.unflatten(-1, (-1, 2)) if interleaved else head.unflatten(-1, (2, -1)).transpose(-1, -2)
    w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
    w = w.flatten(-2) if interleaved else w.transpose(-1, -2).flatten(-2)
    return torch.cat((w, x[..., r:].double()), dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "attend":
        group = case["heads"] // case["kv_heads"]
        outs = []
        for b, n in enumerate(_lengths(case)):  # one sequence at a time
            if n == 0:
                outs.append(torch.zeros(case["heads"], case["dim"], dtype=torch.float64, device="cuda"))
                continue
            held = s["cache"][s["page_table"][b, : -(-n // case["page"])].long()]
            if case["head_major"]:
                held = held.transpose(2, 3)
            k, v = (held[:, i].flatten(0, 1)[:n].double().repeat_interleave(group, dim=1) for i in (0, 1))  # [n, heads, dim]
            weight = torch.softmax(torch.einsum("hd,nhd->hn", s["q"][b].double(), k) / math.sqrt(case["dim"]), dim=-1)
            outs.append(torch.einsum("hn,nhd->hd", weight, v))
        return [torch.stack(outs)]
    if op == "rotary":
        return [_turned(s["x"], s["positions"], s["frequencies"], case["interleaved"], case["inverse"])]
    if op == "append":
        kv_heads = case["kv_heads"]
        k, v = (s["qkv"][:, case["heads"]:].split(kv_heads, dim=1)) if case["packed"] else (s["k"], s["v"])
        kept = s["slots"] >= 0
        flat = s["cache"].double().movedim(1, 0)
        flat = (flat.transpose(2, 3) if case["head_major"] else flat).flatten(1, 2).clone()  # [2, slots, heads, dim]
        flat[0].index_copy_(0, s["slots"][kept].long(), _turned(k, s["positions"], s["frequencies"], False, False)[kept])
        flat[1].index_copy_(0, s["slots"][kept].long(), v[kept].double())
        flat = flat.unflatten(1, (case["pages"], case["page"]))
        return [(flat.transpose(2, 3) if case["head_major"] else flat).movedim(0, 1).contiguous()]
    if op == "norm":
        h = s["x"].double() + (s["residual"].double() if case["residual"] else 0.0)
        y = s["gamma"].double() * h / (h.pow(2).sum(-1, keepdim=True) / case["cols"] + EPS).sqrt()
        more = [h] if case["residual"] else []
        if not case["eight"]:
            return [y] + more
        parts = y.split(case["group"] or case["cols"], dim=-1)
        tops = [p.abs().amax(-1, keepdim=True) for p in parts]
        codes = torch.cat([p * (E4M3_MAX / t) for p, t in zip(parts, tops)], dim=-1)  # the values that the codes round
        return [codes, torch.cat(tops, dim=-1) / E4M3_MAX] + more
    h, dy, gamma, cols = s["h"].double(), s["dy"].double(), s["gamma"].double(), case["cols"]
    norm = (h.pow(2).sum(-1, keepdim=True) / cols + EPS).sqrt()
    inner = (dy * gamma * h).sum(-1, keepdim=True)
    dx = dy * gamma / norm - h * inner / (cols * norm.pow(3))
    return [dx + (s["dsum"].double() if case["residual"] else 0.0), (dy * h / norm).sum(0)]
