"""Workloads of the two ends of a language model, which share one table [vocabulary, columns]: looking tokens up and the
gradient of that, and the cross entropy of hidden states against the table with its gradient.

`listed()` and `draw()` give cases, `prepare()` the data a training or scoring loop has in hand, `run()` one pass through
an operator: in plain torch operations where `own` is false, through the package's public entry points where it is true.
`exact()` evaluates the definition in 64 bits, `work()` counts the bytes and operations a pass cannot do without.
"""
import math

import torch

own = False


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # A decode step of a small batch: one token per sequence, only latency counts.
        dict(name="lookup_step", op="lookup", tokens=16, vocab=32000, cols=4096, padding=0, scaled=False, dtype="bf16"),
        # A prompt against a 32-bit table of odd sizes, scaled by the root of the columns.
        dict(name="lookup_prompt_f32", op="lookup", tokens=2001, vocab=50001, cols=1000, padding=0, scaled=True, dtype="f32"),
        # A training batch, padded behind its sequences.
        dict(name="lookup_batch", op="lookup", tokens=32768, vocab=32000, cols=4096, padding=500, scaled=False, dtype="bf16"),
        # The gradient of a short batch, 32 bits, odd sizes.
        dict(name="lookup_gradient_f32", op="lookup_gradient", tokens=301, vocab=5003, cols=200, padding=7, scaled=True, tied=False, dtype="f32"),
        # The whole table's gradient from a training batch: most of its rows are zeros, a few tokens make up much of the text.
        dict(name="lookup_gradient", op="lookup_gradient", tokens=16384, vocab=32000, cols=4096, padding=300, scaled=False, tied=False, dtype="bf16"),
        # A tied table: the lookup's gradient is added to what the loss has left there.
        dict(name="lookup_gradient_tied", op="lookup_gradient", tokens=32768, vocab=100000, cols=1024, padding=0, scaled=True, tied=True, dtype="bf16"),
        # Scoring the newest token of one sequence: the table is read once, nothing else matters.
        dict(name="score_one", op="score", tokens=1, vocab=32000, cols=4096, ignored=0, dtype="bf16"),
        # Scoring a text in 32 bits, odd sizes.
        dict(name="score_f32", op="score", tokens=999, vocab=10007, cols=1000, ignored=9, dtype="f32"),
        # Scoring a large batch: one matrix product.
        dict(name="score_batch", op="score", tokens=8192, vocab=32000, cols=4096, ignored=100, dtype="bf16"),
        # Loss and gradients of a short sequence, half of which is a prompt that is not learned.
        dict(name="train_small", op="train", tokens=257, vocab=5003, cols=512, ignored=128, dtype="bf16"),
        # Loss and gradients in 32 bits.
        dict(name="train_f32", op="train", tokens=1000, vocab=16001, cols=768, ignored=10, dtype="f32"),
        # Loss and gradients of a training batch.
        dict(name="train_batch", op="train", tokens=8192, vocab=32000, cols=2048, ignored=200, dtype="bf16"),
    ]


def _log_range(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def draw(rng):
    op = rng.choice(["lookup", "lookup_gradient", "lookup_gradient", "score", "score", "train", "train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    size = 2 if dtype == "bf16" else 4
    cols = rng.choice([64, 128, 256, 512, 768, 1024, 2048, 4096, 8 * rng.randint(9, 500), rng.randint(33, 2000)])
    if op in ("lookup", "lookup_gradient"):
        vocab = _log_range(rng, 100, min(131072, (256 << 20) // (cols * size)))
        tokens = _log_range(rng, 1, min(65536, (256 << 20) // (cols * size)))
        case = dict(op=op, tokens=tokens, vocab=vocab, cols=cols, padding=rng.choice([0, rng.randint(0, tokens // 8)]), scaled=rng.random() < 0.5, dtype=dtype)
        return case if op == "lookup" else dict(case, tied=rng.random() < 0.5)
    # 32-bit products cost several of 16 bits
    most = (8192 * 32000 * 2048) // (1 if dtype == "bf16" else 16)
    vocab = _log_range(rng, 50, min(131072, (512 << 20) // (cols * size)))
    tokens = _log_range(rng, 1, max(1, min(8192, most // (vocab * cols), (8192 * 32000) // vocab)))
    return dict(op=op, tokens=tokens, vocab=vocab, cols=cols, ignored=rng.choice([0, rng.randint(0, tokens // 2)]), dtype=dtype)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _scale(case):
    return math.sqrt(case["cols"]) if case.get("scaled") else 1.0


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, op, tokens, vocab, cols = _type(case), case["op"], case["tokens"], case["vocab"], case["cols"]

    def normal(*shape, std=1.0):
        return torch.empty(shape, device="cuda", dtype=t).normal_(0.0, std, generator=g)

    # text: the frequency of a token falls with its number, as in a vocabulary sorted by frequency
    u = torch.rand(tokens, device="cuda", dtype=torch.float64, generator=g)
    ids = (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp_(0, vocab - 1).to(torch.int32)
    s = {"case": dict(case), "ids": ids}
    if op in ("lookup", "lookup_gradient"):
        if case["padding"]:
            ids[tokens - case["padding"]:] = -1
        if op == "lookup":
            s["table"] = normal(vocab, cols, std=0.02)
            s["out"] = torch.empty(tokens, cols, device="cuda", dtype=t)
        else:
            s["dy"] = normal(tokens, cols, std=0.01)
            s["gradient"] = normal(vocab, cols, std=0.01) if case["tied"] else torch.empty(vocab, cols, device="cuda", dtype=t)
        return s
    # a model that has learned something: hidden states lean towards the row of their target
    s["table"] = normal(vocab, cols, std=cols ** -0.5)
    lean = 12.0 * torch.rand(tokens, 1, device="cuda", generator=g)
    s["x"] = (normal(tokens, cols, std=1.5).float() + lean * s["table"][ids.long()].float()).to(t)
    if case["ignored"]:
        ids[torch.randperm(tokens, device="cuda", generator=g)[: case["ignored"]]] = -1
    if op == "train":
        learned = tokens - case["ignored"]
        s["dloss"] = torch.full((tokens,), 1.0 / max(1, learned), device="cuda")
        s["dx"], s["dtable"] = torch.empty_like(s["x"]), torch.empty_like(s["table"])
    s["loss"], s["lse"] = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _lookup(s):
    rows = s["table"][s["ids"].clamp(min=0).long()].float() * _scale(s["case"])
    s["out"].copy_(torch.where((s["ids"] >= 0)[:, None], rows, 0.0))
    return [s["out"]]


def _lookup_gradient(s):
    case = s["case"]
    there = s["ids"] >= 0
    total = torch.zeros(case["vocab"], case["cols"], device="cuda")
    total.index_add_(0, s["ids"].clamp(min=0).long(), torch.where(there[:, None], s["dy"].float(), 0.0))
    total *= _scale(case)
    s["gradient"].copy_(total + s["gradient"].float() if case["tied"] else total)
    return [s["gradient"]]


def _loss(s):
    ids = s["ids"].long()
    there = ids >= 0
    x, table = s["x"].float(), s["table"].float()
    logits = torch.matmul(x, table.t())
    top = logits.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(logits - top).sum(-1, keepdim=True))
    at = ids.clamp(min=0)[:, None]
    s["lse"].copy_(lse[:, 0])
    s["loss"].copy_(torch.where(there, (lse - logits.gather(1, at))[:, 0], 0.0))
    if s["case"]["op"] == "score":
        return [s["loss"], s["lse"]]
    p = torch.exp(logits - lse)
    p.scatter_add_(1, at, torch.full_like(lse, -1.0))
    p *= torch.where(there, s["dloss"], 0.0)[:, None]
    s["dx"].copy_(torch.matmul(p, table))
    s["dtable"].copy_(torch.matmul(p.t(), x))
    return [s["loss"], s["dx"], s["dtable"]]


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

    def use(x):
        handles.append(ctx.from_torch(x))
        return b.input()

    ids = use(s["ids"])
    if op == "lookup":
        b.embedding(use(s["table"]), ids, scale=_scale(case), out=use(s["out"]))
        return ctx, b, handles, [s["out"]]
    if op == "lookup_gradient":
        dy, gradient = use(s["dy"]), use(s["gradient"])
        if case["tied"]:
            b.assign(gradient, b.embedding_grad(dy, ids, case["vocab"], base=gradient, scale=_scale(case)))
        else:
            b.embedding_grad(dy, ids, case["vocab"], scale=_scale(case), out=gradient)
        return ctx, b, handles, [s["gradient"]]
    x, table = use(s["x"]), use(s["table"])
    if op == "score":
        b.vocabulary_loss(x, table, ids, out=[use(s["loss"]), use(s["lse"])])
        return ctx, b, handles, [s["loss"], s["lse"]]
    _, lse = b.vocabulary_loss(x, table, ids, out=[use(s["loss"]), use(s["lse"])])
    b.vocabulary_loss_grad(x, table, ids, lse, use(s["dloss"]), out=[use(s["dx"]), use(s["dtable"])])
    return ctx, b, handles, [s["loss"], s["dx"], s["dtable"]]


def run(state):
    if own:
        if "program" not in state:
            state["program"] = _program(state)
        ctx, step, handles, results = state["program"]
        ctx.record(step, handles)
        ctx.barrier()
        return results
    op = state["case"]["op"]
    return _lookup(state) if op == "lookup" else _lookup_gradient(state) if op == "lookup_gradient" else _loss(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, size, tokens, vocab, cols = case["op"], 2 if case["dtype"] == "bf16" else 4, case["tokens"], case["vocab"], case["cols"]
    if op == "lookup":
        return {"bytes": (2 * tokens - case["padding"]) * cols * size + 4 * tokens, "flops": tokens * cols}
    if op == "lookup_gradient":
        kept = tokens - case["padding"]
        # the rows that are named, where only those change (text as prepare() makes it names about so many)
        chance = math.log(vocab + 1)
        named = min(vocab, sum(1.0 - math.exp(-kept * math.log1p(1.0 / v) / chance) for v in range(1, vocab + 1)))
        return {"bytes": kept * cols * size + (2 * named if case["tied"] else vocab) * cols * size + 4 * tokens, "flops": kept * cols}
    product = 2 * tokens * vocab * cols
    if op == "score":
        return {"bytes": (tokens + vocab) * cols * size + 12 * tokens, "flops": product}
    return {"bytes": 2 * (tokens + vocab) * cols * size + 16 * tokens, "flops": 3 * product}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, ids = case["op"], s["ids"].long()
    if op == "lookup":
        padded = torch.nn.functional.pad(s["table"].double(), (0, 0, 1, 0))  # row 0 stands for no token
        return [torch.nn.functional.embedding(ids + 1, padded) * _scale(case)]
    if op == "lookup_gradient":
        kept = ids[ids >= 0]
        order = torch.argsort(kept, stable=True)
        rows = torch.cumsum(s["dy"][ids >= 0][order].double(), 0)  # differences of running sums: every token of a row at once
        counts = torch.bincount(kept, minlength=case["vocab"])
        ends = torch.cumsum(counts, 0)
        rows = torch.nn.functional.pad(rows, (0, 0, 1, 0))
        total = (rows[ends] - rows[ends - counts]) * _scale(case)
        return [total + s["gradient"].double() if case["tied"] else total]
    x, table = s["x"].double().requires_grad_(op == "train"), s["table"].double().requires_grad_(op == "train")
    logits = torch.nn.functional.linear(x, table)
    loss = torch.nn.functional.cross_entropy(logits, ids, ignore_index=-1, reduction="none")
    if op == "score":
        return [loss, torch.logsumexp(logits, -1)]
    dx, dtable = torch.autograd.grad(loss, (x, table), s["dloss"].double())
    return [loss.detach(), dx, dtable]
