"""The operators that answer with the vocabulary layers, as cases that can be measured: the output layer's logits from weights
and hidden states in 8-bit integers, and the verification of drafted tokens over the sharded logits with the draw of the next one.

``run`` computes a case in its plain form, elementary torch operations in 32 bits (64 where a token hangs on the border between
two), or, where ``own`` is true, through the framework's entry points.  ``exact`` gives the same outputs from the definitions
in 64 bits.

Logits: the hidden states x [N, h] become 8-bit integers row by row, as the weights [V, h] did before,

    s_i = max_j |x_ij| / 127,  q_ij = 127 x_ij / max_j |x_ij| rounded to the nearest integer (ties to even)
    Y_ij = s_i t_j sum_k q_ik w_jk            (w_j, t_j: integers and scale of row j of the weights)

and for every shard of the vocabulary the row maximum, the row sum of exponentials and the label's logit.

Verification: sequence b has the rows starts[b] .. starts[b + 1] - 1 of the logits, one for each of its drafted tokens and one
behind them.  With p_i the target's probabilities in row i and q_i the draft model's (all on the draft itself where there is no
such model), draft d_i is accepted if u_i q_i(d_i) < p_i(d_i) and all before it were.  The next token is drawn from
max(p_i - q_i, 0) of the first rejected row i, or from p of the last row, by the random number of the last row: the first
token at which the running sum exceeds that share of the whole.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
ACCEPTED = 0.75      # about the share of the drafts of these inputs that is accepted


def _logits(name, N, h, V, p, dtype, out):
    # dtype: of the hidden states; out: type of the logits that are kept, "none": the statistics alone
    return {"name": name, "op": "logits", "N": N, "h": h, "V": V, "p": p, "dtype": dtype, "out": out}


def _verify(name, S, K, V, p, dtype, draft, ragged, masked):
    # S sequences of K drafts, or of 0 to K (ragged); draft: the draft model's logits are there; masked: every third token of
    # the vocabulary is ruled out
    return {"name": name, "op": "verify", "S": S, "K": K, "V": V, "p": p, "dtype": dtype, "draft": draft, "ragged": ragged,
            "masked": masked}


def listed():
    return [
        # one new token of one sequence, vocabulary of 128k: latency, and reading the weights
        _logits("logits_token", 1, 4096, 128256, 8, "bf16", "bf16"),
        # eight sequences of four drafts and the row behind them, vocabulary of 32k
        _logits("logits_drafts", 40, 4096, 32000, 8, "bf16", "bf16"),
        # a model in full precision, sizes that are no multiple of anything
        _logits("logits_f32_odd", 509, 1001, 50001, 3, "f32", "f32"),
        # a large batch of single tokens, wide model with a vocabulary of 256k
        _logits("logits_batch", 256, 8192, 256000, 16, "bf16", "bf16"),
        # the loss of a held-out sequence: the statistics alone
        _logits("logits_loss", 4096, 4096, 128256, 8, "bf16", "none"),
        # the wide model's whole context, logits kept
        _logits("logits_wide", 4096, 8192, 256000, 16, "bf16", "bf16"),
        # one sequence and its drafts: latency
        _verify("verify_one", 1, 4, 32000, 8, "bf16", True, False, False),
        # single tokens of a batch, no drafts: sampling
        _verify("sample_batch", 64, 0, 128256, 8, "f32", False, False, False),
        # a batch in the middle of its answers: some sequences have fewer drafts, some none
        _verify("verify_batch", 64, 5, 128256, 8, "bf16", True, True, False),
        # drafts looked up in the text before: no draft model; tokens that a grammar rules out
        _verify("verify_lookup", 32, 8, 50001, 3, "f32", False, True, True),
        # a large batch, vocabulary of 256k
        _verify("verify_large", 256, 8, 256000, 16, "bf16", True, True, False),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    p = rng.choice([1, 2, 3, 4, 8, 16])
    V = _log(rng, 1000, 256000)
    V = V if rng.random() < 0.5 else (V + 127) // 128 * 128
    if rng.random() < 0.5:
        h = _log(rng, 64, 8192)
        h = h if rng.random() < 0.4 else (h + 63) // 64 * 64
        N = rng.choice([1, _log(rng, 2, 64), _log(rng, 2, 4096), _log(rng, 64, 4096)])
        case = _logits("", N, h, V, p, rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "bf16", "f32", "none"]))
    else:
        K = rng.choice([0, rng.randint(1, 4), rng.randint(1, 12)])
        S = rng.choice([1, _log(rng, 2, 64), _log(rng, 2, 256)])
        S = max(1, min(S, 256 * 9 * 256000 // ((K + 1) * V)))
        case = _verify("", S, K, V, p, rng.choice(["bf16", "bf16", "f32"]), K > 0 and rng.random() < 0.7, rng.random() < 0.6,
                       rng.random() < 0.3)
        if case["dtype"] == "f32":
            case["S"] = max(1, S // 2)
    del case["name"]
    return case


def _rows(case):
    """Vocabulary rows of every shard: as even as they get."""
    V, p = case["V"], case["p"]
    return [(r + 1) * V // p - r * V // p for r in range(p)]


def _offsets(case):
    return [r * case["V"] // case["p"] for r in range(case["p"])]


def _counts(case):
    """Drafts of every sequence."""
    return [b * 5 % (case["K"] + 1) if case["ragged"] else case["K"] for b in range(case["S"])]


def _plain_quantize(x):
    a = x.abs().amax(1, keepdim=True)
    # values next to a border: the quotient in 64 bits
    q = torch.round(x.double() * 127 / torch.where(a > 0, a, torch.ones_like(a)).double())
    return q, (a.float() / 127)[:, 0]


def _row_bytes(h):
    return (h + 127) // 128 * 128


def _hidden(case, gen):
    # channels of hidden states differ in size, some by a lot
    x = torch.randn(case["N"], case["h"], generator=gen, device="cuda")
    return (x * torch.exp(0.5 * torch.randn(case["h"], generator=gen, device="cuda"))).to(DTYPES[case["dtype"]])


def _weights(case, gen):
    for n in _rows(case):
        yield torch.randn(n, case["h"], generator=gen, device="cuda") * 0.02


def _prepare_logits(case, gen):
    N, rows = case["N"], _rows(case)
    s = {"x": _hidden(case, gen), "W": [], "W_scales": []}
    for w in _weights(case, gen):
        q, scales = _plain_quantize(w)
        s["W"].append(torch.zeros(w.shape[0], _row_bytes(case["h"]), dtype=torch.int8, device="cuda"))
        s["W"][-1][:, :case["h"]] = q
        s["W_scales"].append(scales)
    s["labels"] = torch.randint(0, case["V"], (N,), generator=gen, device="cuda")
    # where the calls write
    s["q"] = torch.empty(N, _row_bytes(case["h"]), dtype=torch.int8, device="cuda")
    s["scales"] = torch.empty(N, device="cuda")
    s["out"] = {k: torch.empty(case["p"], N, device="cuda") for k in ("max", "sumexp", "target")}
    s["out"]["logits"] = None if case["out"] == "none" else [torch.empty(N, n, dtype=DTYPES[case["out"]], device="cuda") for n in rows]
    return s


def _cut(Y, case, dtype):
    return [y.to(dtype).contiguous() for y in Y.split(_rows(case), 1)]


def _verify_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    counts, V, dt = _counts(case), case["V"], DTYPES[case["dtype"]]
    N = sum(counts) + case["S"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    # a few tokens stand out of a row's many; some rows are surer than others
    Y = normal(N, V).mul_(1.5).mul_(torch.exp(0.3 * normal(N, 1)))
    if case["draft"]:
        Z = Y + 0.5 * normal(N, V)
        if case["masked"]:
            Z[:, ::3] = -math.inf
        Z = Z.to(dt)
        # what the draft model drew
        drafts = (Z - torch.log(-torch.log(torch.rand(N, V, generator=gen, device="cuda").clamp_(1e-7, 1 - 1e-7)))).argmax(1)
    else:
        Z = None
        drafts = torch.randint(0, V // 3, (N,), generator=gen, device="cuda") * 3 + 1
        sure = math.log(V) + 2.5 + normal(N, 1)      # what was looked up is often what the target would say
        Y.scatter_(1, drafts[:, None], sure)
    if case["masked"]:
        Y[:, ::3] = -math.inf
    Y = Y.to(dt)
    starts = torch.tensor([0] + counts).cumsum(0) + torch.arange(case["S"] + 1)
    return {"Y": Y, "Z": Z, "drafts": drafts, "starts": starts.cuda(), "u": torch.rand(N, generator=gen, device="cuda"), "N": N}


def _statistics(Y, case):
    # as the output layer leaves them
    m = Y.amax(1).float()
    return m, sum(torch.exp(y.float() - m[:, None]).sum(1) for y in Y.split(_rows(case), 1))


def prepare(case, seed):
    if case["op"] == "logits":
        return {"case": case, **_prepare_logits(case, torch.Generator(device="cuda").manual_seed(seed))}
    s = {"case": case, **_verify_inputs(case, seed)}
    s["max"], s["sumexp"] = _statistics(s["Y"], case)
    s["draft_max"], s["draft_sumexp"] = _statistics(s["Z"], case) if case["draft"] else (None, None)
    s["logits"] = _cut(s.pop("Y"), case, DTYPES[case["dtype"]])
    Z = s.pop("Z")
    s["draft_logits"] = _cut(Z, case, DTYPES[case["dtype"]]) if case["draft"] else None
    # where the calls write; tokens behind a sequence's next one are -1
    s["accepted"] = torch.empty(case["S"], dtype=torch.int32, device="cuda")
    s["tokens"] = torch.empty(s["N"], dtype=torch.int64, device="cuda")
    return s


# ----------------------------------------------------------------------------------------------- plain forms
def _plain_shard(q, scales, W, W_scales, labels, dtype):
    """One shard's logits (None: not kept) and statistics; labels: within the shard."""
    Y = (q @ W.float().t()) * W_scales * scales[:, None]
    m = Y.amax(1)
    inside = (labels >= 0) & (labels < W.shape[0])
    t = Y.gather(1, labels.clamp(0, W.shape[0] - 1)[:, None])[:, 0]
    kept = None if dtype is None else Y.to(dtype)
    return m, torch.exp(Y - m[:, None]).sum(1), torch.where(inside, t, torch.zeros_like(t)), kept


def _plain_logits(case, s):
    q, scales = _plain_quantize(s["x"])
    q = torch.nn.functional.pad(q.float(), (0, s["W"][0].shape[1] - case["h"]))
    dtype = DTYPES.get(case["out"])
    got = [_plain_shard(q, scales, W, t, s["labels"] - at, dtype) for W, t, at in zip(s["W"], s["W_scales"], _offsets(case))]
    m, e, t, Y = zip(*got)
    return {"max": torch.stack(m), "sumexp": torch.stack(e), "target": torch.stack(t), "logits": None if dtype is None else list(Y)}


def _plain_logit_of(logits, offsets, rows, tokens):
    """The logit of one token in each of these rows."""
    def of(Y, at):
        local = tokens - at
        inside = (local >= 0) & (local < Y.shape[1])
        return torch.where(inside, Y[rows, local.clamp(0, Y.shape[1] - 1)].double(), 0.0)
    return torch.stack([of(Y, at) for Y, at in zip(logits, offsets)]).sum(0)


def _plain_weights(logits, m, e, rows):
    Y = torch.cat([Y[rows] for Y in logits], 1)
    return torch.exp(Y.double() - m[rows, None].double()) / e[rows, None].double()


def _plain_verify(case, s):
    starts, drafts, u, offsets = s["starts"], s["drafts"], s["u"].double(), _offsets(case)
    first, last = starts[:-1], starts[1:] - 1
    # the drafts of all sequences, as many as the longest has
    step = torch.arange(max(1, case["K"]), device="cuda")
    rows = torch.minimum(first[:, None] + step, last[:, None])
    is_draft = first[:, None] + step < last[:, None]
    d = drafts[rows]
    p = torch.exp(_plain_logit_of(s["logits"], offsets, rows, d) - s["max"][rows].double()) / s["sumexp"][rows].double()
    if case["draft"]:
        q = torch.exp(_plain_logit_of(s["draft_logits"], offsets, rows, d) - s["draft_max"][rows].double())
        q = q / s["draft_sumexp"][rows].double()
    else:
        q = torch.ones_like(p)
    accepted = (is_draft & (u[rows] * q < p)).long().cumprod(1).sum(1)
    # the next token
    row = first + accepted
    rejected = (row < last)[:, None]
    w = _plain_weights(s["logits"], s["max"], s["sumexp"], row)
    if case["draft"]:
        w = w - torch.where(rejected, _plain_weights(s["draft_logits"], s["draft_max"], s["draft_sumexp"], row), 0.0)
    else:
        w = w.scatter(1, drafts[row, None], torch.where(rejected, 0.0, w.gather(1, drafts[row, None])))
    c = w.clamp_(min=0).cumsum(1)
    token = (c <= u[last][:, None] * c[:, -1:]).sum(1)
    # accepted drafts, the next token, -1 behind it
    at = torch.arange(s["N"], device="cuda")
    b = torch.searchsorted(starts, at, right=True) - 1
    behind = at - row[b]
    return {"accepted": accepted.int(), "tokens": torch.where(behind < 0, drafts, torch.where(behind == 0, token[b], -1))}


# ----------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        return _own(case, s)
    return _plain_logits(case, s) if case["op"] == "logits" else _plain_verify(case, s)


def _own(case, s):
    import paper_2411_05288_amd as vp
    if case["op"] == "logits":
        if "workspace" not in s:      # once for these sizes
            n = vp.vp_output_i8_workspace_bytes(case["N"], _rows(case))
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        out = s["out"]
        vp.vp_quantize_rows(s["x"], s["q"], s["scales"])
        vp.vp_output_fwd_i8_group(s["q"], s["scales"], s["W"], s["W_scales"], s["labels"], _offsets(case), out["max"],
                                  out["sumexp"], out["target"], out["logits"], workspace=s["workspace"])
        return out
    if "workspace" not in s:
        s["workspace"] = torch.empty(vp.vp_verify_workspace_bytes(case["S"], case["V"]), dtype=torch.uint8, device="cuda")
    vp.vp_verify_drafts(s["logits"], _offsets(case), s["max"], s["sumexp"], s["drafts"], s["starts"], s["u"], s["accepted"],
                        s["tokens"], s["workspace"], draft_logits=s["draft_logits"], draft_max=s["draft_max"],
                        draft_sumexp=s["draft_sumexp"])
    return {"accepted": s["accepted"], "tokens": s["tokens"]}


# ----------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    V, e = case["V"], BYTES[case["dtype"]]
    if case["op"] == "logits":
        N, h = case["N"], case["h"]
        return {"bytes": N * h * e + V * h + 4 * V + 12 * N * case["p"] + 8 * N + N * V * BYTES.get(case["out"], 0),
                "flops": 2 * N * h * V}
    # one row of every sequence, and the draft model's row where a draft was rejected; an exponential, a difference and a sum
    # of each
    rows = sum(1 + case["draft"] * (1 - ACCEPTED ** k) for k in _counts(case))
    return {"bytes": int(rows * V * e) + 24 * (sum(_counts(case)) + case["S"]), "flops": int(rows * V * 20)}


# ----------------------------------------------------------------------------------------------- in 64 bits
def _exact_integers(x):
    """127 x / max |x| to the nearest integer: its whole part, and one more where what is left is more than half, or half of an odd one."""
    x = x.double()
    largest = x.abs().max(1, keepdim=True).values
    t = 127 * x.abs() / largest
    whole = t.floor()
    up = (t - whole > 0.5) | ((t - whole == 0.5) & (whole.remainder(2) == 1))
    return (whole + up) * x.sign(), largest / 127


def _exact_logits(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, scale = _exact_integers(_hidden(case, gen))
    out = {"max": [], "sumexp": [], "target": [], "logits": []}
    integers = [_exact_integers(w) for w in _weights(case, gen)]
    integers = [(w.to(torch.int8), t) for w, t in integers]
    labels = torch.randint(0, case["V"], (case["N"],), generator=gen, device="cuda")
    for (w, t), at in zip(integers, _offsets(case)):
        # (the scales that a call gets are rounded to 32 bits)
        Y = torch.mm(scale.float().double() * q, (w.double() * t.float().double()).t().contiguous())
        out["max"].append(Y.max(1).values)
        out["sumexp"].append((Y - out["max"][-1][:, None]).exp().sum(1))
        hit = torch.arange(at, at + w.shape[0], device="cuda")[None, :] == labels[:, None]
        out["target"].append(Y.masked_fill(~hit, 0).sum(1))
        if case["out"] != "none":
            out["logits"].append(Y)
    return {k: (torch.stack(v) if k != "logits" else v or None) for k, v in out.items()}


def _exact_verify(case, seed):
    """Row by row, by the inverse of the distribution function."""
    s = _verify_inputs(case, seed)
    m, e = _statistics(s["Y"], case)
    p = lambda i: torch.exp(s["Y"][i].double() - m[i].double()) / e[i].double()      # noqa: E731
    if case["draft"]:
        mz, ez = _statistics(s["Z"], case)
    starts, tokens, counts = s["starts"].tolist(), [], []
    drafts, u = s["drafts"].tolist(), s["u"].tolist()
    for b in range(case["S"]):
        i, last = starts[b], starts[b + 1] - 1
        while True:
            weights = p(i)
            if i == last:
                break
            q = torch.zeros_like(weights)
            q[drafts[i]] = 1
            if case["draft"]:
                q = torch.exp(s["Z"][i].double() - mz[i].double()) / ez[i].double()
            if not u[i] * float(q[drafts[i]]) < float(weights[drafts[i]]):
                weights = (weights - q).relu()
                break
            i += 1
        c = weights.cumsum(0)
        token = int(torch.searchsorted(c, u[last] * c[-1], right=True))
        counts.append(i - starts[b])
        tokens += drafts[starts[b]:i] + [token] + [-1] * (last - i)
    return {"accepted": torch.tensor(counts, dtype=torch.int32), "tokens": torch.tensor(tokens)}


def exact(case, seed):
    return _exact_logits(case, seed) if case["op"] == "logits" else _exact_verify(case, seed)
