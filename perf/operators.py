"""Operators of the model update: a matrix orthogonalised by Newton-Schulz products, the update through it, and AdamW.

The framework's flat vector [d] holds a model's matrices (and what is no matrix between them).  A case is a dict of plain
values:
  op        'orthogonalize'  every matrix of a flat vector, on its own
            'update_ortho'   the server's message through momentum and the matrices' orthogonalisation into the model
            'update_adamw'   the server's message through two moments into the model, everything but the matrices
  mats      the matrices in their order: 'RxC', 'RxC*N' for N of them, 'RxC/P' for P column blocks of one stored RxC array;
            '' for none
  gap       elements between one matrix and the next      d   elements of the vector, 0: as many as the matrices need
  dtype     orthogonalize: 'f32' or 'bf16' in and out.  f32 takes products of fp32 grade, bf16 single half-precision products
  comp      the message: 'identity', 'sign' (one scale per chunk), 'topk', 'qsgd';  chunk, k, bucket, levels: their sizes
  scale     factor of an orthogonalised matrix: 'none', 'aspect' = sqrt(max(1, rows / cols)), 'rms' = 0.2 sqrt(max(rows, cols))
  nesterov, decay, steps
"""
from __future__ import annotations

import math
import random

import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)
NORM_EPS = 1e-7
GAMMA, BETA = 0.02, 0.95
ADAM_GAMMA, BETA1, BETA2, ADAM_EPS, ADAM_STEP = 1e-3, 0.9, 0.95, 1e-8, 7
GPT2_SMALL = 124_439_808          # the vector of the repository's largest workload
RESNET50 = 25_557_032
BLOCKS = "768x2304*12,768x768*12,768x2048*24,2048x768*12"    # twelve blocks of width 768 with a gated MLP
MOST_FLOPS = 1.0e12
MOST_ELEMENTS = 100_000_000


def _resnet50():
    """The convolutions of ResNet-50 as [out, in * kh * kw] matrices, and its classifier."""
    mats, width = ["64x147"], 64
    for planes, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
        for i in range(blocks):
            mats += [f"{planes}x{width}", f"{planes}x{9 * planes}", f"{4 * planes}x{planes}"]
            if i == 0:
                mats.append(f"{4 * planes}x{width}")
            width = 4 * planes
    return ",".join(mats + ["1000x2048"])


def _case(name, op, mats="", **more):
    c = {"op": op, "mats": mats, "gap": 0, "d": 0, "dtype": "f32", "comp": "identity", "chunk": 0, "k": 0, "bucket": 0,
         "levels": 0, "scale": "none", "nesterov": False, "decay": 0.0, "steps": 5}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one small layer: nothing but the latency of a chain of dependent products
        _case("ortho_f32_96x64", "orthogonalize", "96x64"),
        # odd and thin matrices, a row vector, three column blocks of one array, at odd offsets
        _case("ortho_f32_ragged", "orthogonalize", "333x1001,1000x77,1x513,96x480/3,257x255,70x1,640x641", gap=3),
        # the largest square layer of a medium model
        _case("ortho_f32_4096x4096", "orthogonalize", "4096x4096"),
        # all layers of a small model at once, held in bf16 as its gradients are
        _case("ortho_bf16_blocks768", "orthogonalize", BLOCKS, dtype="bf16"),
        # a wide projection in bf16
        _case("ortho_bf16_2048x8192", "orthogonalize", "2048x8192", dtype="bf16"),
        # a step of a toy model: the uncompressed message, a few small layers
        _case("update_ortho_small", "update_ortho", "64x48*3,32x64", gap=8, comp="identity", nesterov=True),
        # ResNet-50, every convolution as a matrix, from a top-k message; norms and biases lie between the layers
        _case("update_ortho_resnet50_topk", "update_ortho", _resnet50(), gap=992, d=RESNET50, comp="topk", k=RESNET50 // 100,
              scale="aspect", nesterov=True),
        # the largest workload: 1-bit message of the whole model, its sixty matrices updated
        _case("update_ortho_124m_sign", "update_ortho", BLOCKS, gap=832, d=GPT2_SMALL, comp="sign", chunk=2048, scale="rms",
              nesterov=True, decay=0.1),
        # the smallest AdamW step: latency
        _case("adamw_sign_1k", "update_adamw", d=1024, comp="sign", chunk=512),
        # what is no convolution of ResNet-50 is skipped over: an update of everything but the matrices
        _case("adamw_resnet50_qsgd_skip", "update_adamw", _resnet50(), gap=992, d=RESNET50, comp="qsgd", bucket=512, levels=15,
              decay=0.01),
        # AdamW of a whole model of odd length from a top-k message
        _case("adamw_11m_topk", "update_adamw", d=11_173_961, comp="topk", k=111_739),
        # AdamW of the largest workload's vector from its 1-bit message
        _case("adamw_124m_sign", "update_adamw", d=GPT2_SMALL, comp="sign", chunk=2048, decay=0.1),
    ]


def _flops(r, c, steps):
    m, n = min(r, c), max(r, c)
    return steps * (3 * m * m * n + m * m * m)


def draw(rng: random.Random):
    """One more case of the same ranges: vectors and matrices from single elements up to the largest listed ones."""
    op = rng.choice(["orthogonalize", "orthogonalize", "update_ortho", "update_ortho", "update_adamw"])

    def size(hi):
        s = int(math.exp(rng.uniform(0.0, math.log(hi + 0.5))))
        return max(1, s - s % 64 if s >= 128 and rng.random() < 0.5 else s)

    mats, flops, total = [], 0, 0
    for _ in range(rng.choice([1, 1, 2, 3, 5, 8, 13, 24])):
        r, c = size(4096), size(8192)
        if rng.random() < 0.5:
            r, c = c, r
        if flops + _flops(r, c, 5) <= MOST_FLOPS and total + r * c <= MOST_ELEMENTS:
            mats.append(f"{r}x{c}")
            flops, total = flops + _flops(r, c, 5), total + r * c
    c = _case(None, op, ",".join(mats or ["64x96"]), gap=rng.choice([0, 0, 1, 2, 5, 64, 1000]))
    c["steps"] = rng.choice([1, 3, 5, 5, 5, 6])
    if c["steps"] == 6:
        c["steps"] = 5 if flops > MOST_FLOPS * 0.8 else 6
    c["scale"] = rng.choice(["none", "aspect", "rms"])
    if op == "orthogonalize":
        c["dtype"] = rng.choice(["f32", "bf16"])
        return c
    if op == "update_adamw" and rng.random() < 0.5:
        c["mats"], c["gap"] = "", 0
        c["d"] = size(GPT2_SMALL) + 3
    if c["mats"] and op == "update_adamw":
        c["gap"] = max(c["gap"], 64)              # there is something beside the matrices
    d = c["d"] or _layout(c)[1]
    c["comp"] = rng.choice(["identity", "sign", "topk", "qsgd"])
    c["chunk"] = rng.choice([512, 2048, 2048]) if c["comp"] == "sign" else 0
    c["k"] = max(1, d // rng.choice([10, 100, 1000])) if c["comp"] == "topk" else 0
    c["bucket"], c["levels"] = rng.choice([(64, 7), (128, 15), (512, 15)]) if c["comp"] == "qsgd" else (0, 0)
    c["nesterov"] = rng.random() < 0.6
    c["decay"] = rng.choice([0.0, 0.01, 0.1])
    return c


def _layout(case):
    """[(offset, rows, cols, row stride)] of the matrices, and the length of the vector."""
    out, at = [], 0
    for item in filter(None, case["mats"].split(",")):
        body, _, count = item.partition("*")
        shape, _, parts = body.partition("/")
        r, c = (int(v) for v in shape.split("x"))
        parts = int(parts or 1)
        for _ in range(int(count or 1)):
            for p in range(parts):
                out.append((at + p * (c // parts), r, c // parts, c))
            at += r * c + case["gap"]
    return out, max(case["d"], at, 1)


def _rows_of(flat, mat):
    offset, r, c, ld = mat
    return flat.as_strided((r, c), (ld, 1), offset)


def _gradient_like(case, mats, d, gen):
    """Noise with a few strong directions in every matrix and layers of different magnitude, as gradients have."""
    g = torch.randn(d, generator=gen, device="cuda").mul_(1e-3)
    for i, mat in enumerate(mats):
        view = _rows_of(g, mat)
        r, c = view.shape
        left = torch.randn(r, 6, generator=gen, device="cuda")
        right = torch.randn(6, c, generator=gen, device="cuda")
        view.add_(left @ right, alpha=3e-4).mul_(10.0 ** (-(i % 4)))
    return g


def _message(case, d, gen):
    """The server's message in the layout of include/ds.h, as a worker receives it."""
    comp = case["comp"]
    if comp == "identity":
        return {"dense": torch.randn(1, d, generator=gen, device="cuda").mul_(1e-3)}
    if comp == "topk":
        idx = torch.randperm(d, generator=gen, device="cuda")[:case["k"]].sort().values.to(torch.int32)
        val = torch.randn(case["k"], generator=gen, device="cuda").mul_(1e-2)
        return {"pairs": torch.stack([idx, val.view(torch.int32)], dim=1).reshape(1, case["k"], 2).contiguous()}
    words = (d + 63) // 64
    bits = torch.randint(0, 1 << 32, (words, 2), generator=gen, device="cuda", dtype=torch.int64)
    plane = bits[:, 0] | (bits[:, 1] << 32)
    if d % 64:
        plane[-1] &= (1 << (d % 64)) - 1
    group = case["chunk"] if comp == "sign" else case["bucket"]
    scales = torch.rand(1, (d + group - 1) // group, generator=gen, device="cuda").add_(0.5).mul_(1e-3)
    if comp == "sign":
        return {"sign_words": plane.reshape(1, words), "scales": scales}
    codes = torch.randint(0, case["levels"] + 1, (d + d % 2,), generator=gen, device="cuda", dtype=torch.uint8)
    codes[d:] = 0
    return {"sign_words": plane.reshape(1, words), "scales": scales.mul_(20.0),
            "levels": (codes[0::2] | (codes[1::2] << 4)).reshape(1, -1).contiguous()}


def _inputs(case, seed):
    mats, d = _layout(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * (int(seed) + 1) + 11)
    s = {"case": case, "mats": mats, "d": d}
    if case["op"] == "orthogonalize":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s["src"] = _gradient_like(case, mats, d, gen).to(dtype)
        s["dst"] = torch.zeros(d, dtype=dtype, device="cuda")
        return s
    s["msg"] = _message(case, d, gen)
    s["x"] = torch.randn(d, generator=gen, device="cuda").mul_(0.02)
    s["m"] = _gradient_like(case, mats, d, gen).mul_(5.0)
    if case["op"] == "update_adamw":
        s["v"] = torch.rand(d, generator=gen, device="cuda").add_(0.05).mul_(1e-6)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_1905_05957_amd as P
        s["plan"] = P.OrthoPlan(s["d"], s["mats"], steps=case["steps"], coef=COEF, eps=NORM_EPS, scale=case["scale"],
                                nesterov=case["nesterov"], half=case["dtype"] == "bf16") if s["mats"] else None
        if "msg" in s:
            s["ctx"] = P.Context(case["comp"], 1, s["d"], scale_mode="chunk" if case["comp"] == "sign" else "whole",
                                 chunk=case["chunk"], k=case["k"], bucket=case["bucket"] or 512, levels=case["levels"] or 15)
            s["srv"] = s["ctx"].alloc_payload(1)
            for name, t in s["srv"].tensors().items():
                t.copy_(s["msg"][name])
    return s


# ---------------------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------------------
def _factor(case, r, c):
    return {"none": 1.0, "aspect": math.sqrt(max(1.0, r / c)), "rms": 0.2 * math.sqrt(max(r, c))}[case["scale"]]


def _orthogonal(case, u):
    """The polynomial iteration on one matrix in fp32; the norm is a long sum: 64 bits."""
    a, b, c = COEF
    flip = u.shape[0] > u.shape[1]
    x = u.t() if flip else u
    norm = x.double().square().sum().sqrt() + NORM_EPS
    x = (x.double() / norm).float()
    for _ in range(case["steps"]):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    x = x * _factor(case, *u.shape)
    return x.t() if flip else x


def _decode(case, msg, d):
    comp = case["comp"]
    if comp == "identity":
        return msg["dense"][0]
    if comp == "topk":
        q = torch.zeros(d, device="cuda")
        q[msg["pairs"][0, :, 0].long()] = msg["pairs"][0, :, 1].contiguous().view(torch.float32)
        return q
    bit = torch.arange(64, device="cuda")
    negative = ((msg["sign_words"][0].unsqueeze(1) >> bit) & 1).to(torch.bool).reshape(-1)[:d]
    group = case["chunk"] if comp == "sign" else case["bucket"]
    size = torch.repeat_interleave(msg["scales"][0], group)[:d]
    if comp == "qsgd":
        byte = msg["levels"][0]
        code = torch.stack([byte & 15, byte >> 4], dim=1).reshape(-1)[:d]
        size = code.float() * (size / case["levels"])
    return torch.where(negative, -size, size)


def _outside(mats, d):
    keep = torch.ones(d, dtype=torch.bool, device="cuda")
    for mat in mats:
        _rows_of(keep, mat).fill_(False)
    return keep


def _run_plain(s):
    case, mats, d = s["case"], s["mats"], s["d"]
    if case["op"] == "orthogonalize":
        for mat in mats:
            _rows_of(s["dst"], mat).copy_(_orthogonal(case, _rows_of(s["src"], mat).float()))
        return s["dst"]
    q = _decode(case, s["msg"], d)
    if case["op"] == "update_ortho":
        for mat in mats:
            qm, mm, xm = (_rows_of(t, mat) for t in (q, s["m"], s["x"]))
            mm.mul_(BETA).add_(qm)
            u = BETA * mm + qm if case["nesterov"] else mm
            xm.mul_(1.0 - GAMMA * case["decay"]).sub_(GAMMA * _orthogonal(case, u))
        return {"x": s["x"], "m": s["m"]}
    m = BETA1 * s["m"] + (1.0 - BETA1) * q
    v = BETA2 * s["v"] + (1.0 - BETA2) * (q * q)
    size = (v / (1.0 - BETA2 ** (ADAM_STEP + 1))).sqrt() + ADAM_EPS
    x = s["x"] * (1.0 - ADAM_GAMMA * case["decay"]) - ADAM_GAMMA * (m / (1.0 - BETA1 ** (ADAM_STEP + 1))) / size
    if mats:
        keep = _outside(mats, d)
        m, v, x = (torch.where(keep, new, s[name]) for name, new in (("m", m), ("v", v), ("x", x)))
    for name, new in (("m", m), ("v", v), ("x", x)):
        s[name].copy_(new)
    return {"x": s["x"], "m": s["m"], "v": s["v"]}


def run(state):
    if not own:
        return _run_plain(state)
    case, op = state["case"], state["case"]["op"]
    if op == "orthogonalize":
        state["plan"].orthogonalize(state["src"], state["dst"])
        return state["dst"]
    if op == "update_ortho":
        state["ctx"].apply_update_ortho(state["plan"], state["srv"], state["x"], state["m"], GAMMA, BETA, decay=case["decay"])
        return {"x": state["x"], "m": state["m"]}
    state["ctx"].apply_update_adamw(state["srv"], ADAM_STEP, state["x"], state["m"], state["v"], ADAM_GAMMA, BETA1, BETA2,
                                    ADAM_EPS, decay=case["decay"], skip=state["plan"])
    return {"x": state["x"], "m": state["m"], "v": state["v"]}


def work(case):
    """Every input read once, every output written once; products of which one half follows by symmetry count as half."""
    mats, d = _layout(case)
    inside = sum(r * c for _, r, c, _ in mats)
    flops = sum(_flops(r, c, case["steps"]) for _, r, c, _ in mats)
    if case["op"] == "orthogonalize":
        return {"bytes": inside * (4 if case["dtype"] == "bf16" else 8), "flops": flops + 3 * inside}
    touched = inside if case["op"] == "update_ortho" else d - inside
    share = touched / d
    message = {"identity": 4 * touched, "topk": 8 * case["k"] * share, "sign": touched / 8 + 4 * touched / max(1, case["chunk"]),
               "qsgd": touched * 5 / 8 + 4 * touched / max(1, case["bucket"])}[case["comp"]]
    if case["op"] == "update_ortho":
        return {"bytes": int(message) + 16 * touched, "flops": flops + 10 * touched}
    return {"bytes": int(message) + 24 * touched, "flops": 14 * touched}


# ---------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------
def _polar_step_64(y, a, b, c):
    """a Y + b (Y Y') Y + c (Y Y')^2 Y on the shorter side's Gram matrix."""
    if y.shape[0] <= y.shape[1]:
        gram = torch.mm(y, y.t().contiguous())
        once = torch.mm(gram, y)
        return a * y + b * once + c * torch.mm(gram, once)
    gram = torch.mm(y.t().contiguous(), y)
    once = torch.mm(y, gram)
    return a * y + b * once + c * torch.mm(once, gram)


def _block_64(flat, mat):
    start, r, c, ld = mat
    index = torch.arange(r, device="cuda").unsqueeze(1) * ld + torch.arange(c, device="cuda") + start
    return index, flat[index]


def _matrix_64(case, u):
    y = u / (torch.sqrt((u * u).sum()) + NORM_EPS)
    for _ in range(case["steps"]):
        y = _polar_step_64(y, *COEF)
    r, c = u.shape
    if case["scale"] == "aspect":
        return y * math.sqrt(r / c) if r > c else y
    return y * (0.2 * math.sqrt(max(r, c))) if case["scale"] == "rms" else y


def _values_64(case, msg, d):
    at = torch.arange(d, device="cuda")
    if case["comp"] == "identity":
        return msg["dense"].reshape(-1).double()
    if case["comp"] == "topk":
        out = torch.zeros(d, dtype=torch.float64, device="cuda")
        return out.index_put((msg["pairs"][0, :, 0].long(),), msg["pairs"][0, :, 1].contiguous().view(torch.float32).double())
    sign = 1.0 - 2.0 * ((msg["sign_words"].reshape(-1)[at // 64] >> (at % 64)) & 1).double()
    if case["comp"] == "sign":
        return sign * msg["scales"].reshape(-1)[at // case["chunk"]].double()
    code = (msg["levels"].reshape(-1)[at // 2].long() >> (4 * (at % 2))) & 15
    return sign * code.double() * msg["scales"].reshape(-1)[at // case["bucket"]].double() / case["levels"]


def exact(case, seed):
    s = _inputs(case, seed)
    mats, d = s["mats"], s["d"]
    if case["op"] == "orthogonalize":
        src, out = s["src"].double(), torch.zeros(d, dtype=torch.float64, device="cuda")
        for mat in mats:
            index, u = _block_64(src, mat)
            out[index] = _matrix_64(case, u)
        return out
    q, x, m = _values_64(case, s["msg"], d), s["x"].double(), s["m"].double()
    if case["op"] == "update_ortho":
        for mat in mats:
            index, qm = _block_64(q, mat)
            new = BETA * m[index] + qm
            m[index] = new
            u = BETA * new + qm if case["nesterov"] else new
            x[index] = x[index] * (1.0 - GAMMA * case["decay"]) - GAMMA * _matrix_64(case, u)
        return {"x": x, "m": m}
    v = s["v"].double()
    touched = torch.ones(d, dtype=torch.bool, device="cuda")
    for mat in mats:
        touched[_block_64(q, mat)[0]] = False
    at = touched.nonzero().reshape(-1)
    qa = q[at]
    m[at] = BETA1 * m[at] + (1.0 - BETA1) * qa
    v[at] = BETA2 * v[at] + (1.0 - BETA2) * qa ** 2
    mean, square = m[at] / (1.0 - BETA1 ** (ADAM_STEP + 1)), v[at] / (1.0 - BETA2 ** (ADAM_STEP + 1))
    x[at] -= ADAM_GAMMA * (mean / (square.sqrt() + ADAM_EPS) + case["decay"] * x[at])
    return {"x": x, "m": m, "v": v}
