"""Rotary positions, and rows into and out of the 4-bit cache, against the 64-bit oracle.

Tolerances.  The rotation takes two products and a sum of inputs in fp32 (3 roundings of 2^-24 of |a| + |b|) with factors
rounded to fp32 (2^-24 each), then the output type's rounding (8, 11 or 24 significant bits: 2^-8, 2^-11 or 2^-24 of the result): at most
u |y| + 2^-21 (|a| + |b|).  Codes, scales and centres of rows that are not rotated are the format's to the bit; of rotated
rows a value may lie a code off where the rotation's rounding meets a code's edge: each value is within one step of its
group (15 steps to the group's spread) of the input, and within half a step but for such edges.
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
UNIT = {BF16: 2.0 ** -8, FP16: 2.0 ** -11, FP32: 2.0 ** -24}
THETA = 1e6


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


def _kv4():
    from paper_2609_34045_gb300 import kv4
    return kv4


def freqs(r, theta=THETA):
    return theta ** (-np.arange(0, r, 2) / r)


def int32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def randn(shape, dtype, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def near(got, ref, a_plus_b):
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= UNIT[got.dtype] * np.abs(ref) + 2.0 ** -21 * a_plus_b + 2.0 ** -40).all(), float(err.max())


# ---- rotation

@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,r,heads,kv", [(128, 128, 28, 4), (64, 64, 8, 2), (128, 64, 64, 8), (128, 32, 3, 1), (80, 20, 5, 2),
                                           (96, 96, 2, 1), (2, 2, 1, 1), (512, 512, 2, 1), (512, 2, 1, 1), (126, 36, 3, 3)])
@pytest.mark.parametrize("n", [1, 7, 700])
def test_rotation(hd, r, heads, kv, layout, dtype, n):
    kv4 = _kv4()
    table = kv4.kfl_rope_table(5000, r, THETA)
    x = randn((n, heads + 2 * kv, hd), dtype, seed=n + hd)  # a fused projection: strided views
    q, k = x[:, :heads], x[:, heads:heads + kv]
    pos = np.random.default_rng(n).integers(0, 5000, n)
    q_out, k_out = torch.empty(n, heads, hd, dtype=dtype, device="cuda"), torch.empty(n, kv, hd, dtype=dtype, device="cuda")
    kv4.kfl_rope(kv4.rope_plan(table, layout), q, q_out, k, k_out, int32(pos))
    angles = pos[:, None] * freqs(r)
    for a, b in ((q, q_out), (k, k_out)):
        ref = ora.rotate(a.double().cpu().numpy(), angles, layout == "interleaved")
        near(b, ref, np.abs(a.double().cpu().numpy()).max(-1, keepdims=True) * 2)
        assert torch.equal(b[..., r:], a[..., r:])
    # in place, odd strides, q alone: the same bits
    wide = torch.zeros(n, heads, hd + 3, dtype=dtype, device="cuda")[..., 3:]
    wide.copy_(q)
    kv4.kfl_rope(kv4.rope_plan(table, layout), wide, wide, None, None, int32(pos))
    assert torch.equal(wide, q_out)


def test_rotation_of_no_tokens_and_of_bad_positions():
    kv4 = _kv4()
    plan = kv4.rope_plan(kv4.kfl_rope_table(10, 64, THETA))
    q = randn((3, 2, 64), BF16)
    out, status = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kfl_rope(plan, q[:0], out[:0], None, None, int32([]))
    kv4.kfl_rope(plan, q, out, None, None, int32([10, 9, -1]), status=status)
    assert status.item() == kv4.KFL_BAD_POSITION
    assert (out[0] == 7).all() and (out[2] == 7).all() and not (out[1] == 7).any()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_the_inverse_is_the_gradient(layout):
    """The rotation is linear: its gradient is the transposed matrix, taken here from the formula (unit vectors through
    the oracle) and from differences of the operator itself."""
    kv4 = _kv4()
    r, hd, n = 32, 48, 5
    plan = kv4.rope_plan(kv4.kfl_rope_table(100, r, 1e4), layout)
    pos = np.array([0, 1, 17, 50, 99])
    dy, x, dx = randn((n, 2, hd), FP32, 1), randn((n, 2, hd), FP32, 2), torch.empty(n, 2, hd, device="cuda")
    kv4.kfl_rope(plan, dy, dx, None, None, int32(pos), inverse=True)
    angles = pos[:, None] * freqs(r, 1e4)
    matrix = ora.rotate(np.broadcast_to(np.eye(hd), (n, hd, hd)), angles, layout == "interleaved")  # [token][in][out]
    near(dx, np.einsum("tio,tho->thi", matrix, dy.double().cpu().numpy()), np.full((n, 2, 1), 8.0))
    loss = []
    d = randn((n, 2, hd), FP32, 3)
    for eps in (1.0, -1.0):  # (exact for a linear operator but for rounding: a large step)
        y = torch.empty_like(x)
        kv4.kfl_rope(plan, x + eps * d, y, None, None, int32(pos))
        loss.append((y.double() * dy.double()).sum().item())
    assert abs((loss[0] - loss[1]) / 2 - (dx.double() * d.double()).sum().item()) < 1e-3


@pytest.mark.parametrize("cfg", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                 dict(scaling="bands", factor=8.0, low=1.0, high=4.0, original_ctx=8192.0),
                                 dict(scaling="ramp", factor=16.0, low=1.0, high=32.0, original_ctx=4096.0),
                                 dict(scaling="ramp", factor=16.0, low=1.0, high=32.0, original_ctx=4096.0, magnitude=0.5),
                                 dict(scaling="plain", magnitude=2.0)])
def test_tables_for_long_contexts(cfg):
    kv4 = _kv4()
    r, theta = 128, 5e5
    got = kv4.kfl_rope_table(3000, r, theta, **cfg).double().cpu().numpy()
    f = freqs(r, theta)
    kind, s, m = cfg["scaling"], cfg.get("factor", 1.0), cfg.get("magnitude", 0.0) or 1.0
    if kind == "linear":
        f = f / s
    elif kind == "base":
        f = freqs(r, theta * s ** (r / (r - 2)))
    elif kind == "bands":
        keep = np.clip((cfg["original_ctx"] / (2 * np.pi / f) - cfg["low"]) / (cfg["high"] - cfg["low"]), 0, 1)
        f = keep * f + (1 - keep) * f / s
    elif kind == "ramp":
        at = [r * np.log(cfg["original_ctx"] / (2 * np.pi * b)) / (2 * np.log(theta)) for b in (cfg["high"], cfg["low"])]
        a, b = max(np.floor(at[0]), 0), min(np.ceil(at[1]), r - 1)
        ramp = np.clip((np.arange(r // 2) - a) / (b - a), 0, 1)
        f = f * (1 - ramp) + f / s * ramp
        m = cfg.get("magnitude", 0.0) or 0.1 * np.log(s) + 1
    angle = np.arange(3000)[:, None] * f
    ref = m * np.stack([np.cos(angle), np.sin(angle)], -1)
    # fp32's rounding, and the angles' own (3000 positions in 64 bits)
    assert np.abs(got - ref).max() <= m * 2.0 ** -24 + 1e-11


# ---- rows of the cache

def cache(lengths, kv, hd, page, layers=1, extra=1):
    kv4 = _kv4()
    need = [-(-n // page) for n in lengths]
    order = np.random.default_rng(1).permutation(sum(need) + 2).astype(np.int32)
    table = np.full((len(lengths), max(need) + extra), -1, dtype=np.int32)
    at = 0
    for u, n in enumerate(need):
        table[u, :n] = order[at:at + n]
        at += n
    pool_t = torch.full((sum(need) + 2, layers, kv, page * hd * 9 // 8), 255, dtype=torch.uint8, device="cuda")
    m = kv4.page_map(int32(table), int32(lengths), torch.zeros(sum(need) + 2, dtype=torch.int32, device="cuda"))
    return kv4, pool_t, kv4.pool(pool_t, page, layers, kv, hd), m, table


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("hd,kv,page,layers", [(128, 8, 64, 1), (128, 1, 16, 3), (64, 2, 32, 2), (64, 3, 128, 1)])
@pytest.mark.parametrize("lengths", [[1], [1, 33, 200, 64]])
def test_append_and_read(hd, kv, page, layers, lengths, dtype):
    kv4, pool_t, p, m, table = cache(lengths, kv, hd, page, layers)
    users = np.concatenate([[u] * n for u, n in enumerate(lengths)])
    pos = np.concatenate([np.arange(n) for n in lengths])
    order = np.random.default_rng(2).permutation(len(users))
    users, pos = users[order], pos[order]
    x = randn((len(users), 2 * kv, hd), dtype, seed=3) * 3
    k, v = x[:, :kv], x[:, kv:]
    layer = layers - 1
    before = pool_t.clone()
    kv4.kfl_kv4_append(p, m, layer, k, v, int32(users), int32(pos))
    # every byte of the written rows as the format has it, every other byte as it was
    want = before.cpu().numpy()
    n, par = page * hd // 2, page * hd // 16
    for i, rows in enumerate((k, v)):
        codes, params = ora.quantise(rows.float().cpu().numpy())
        packed = codes[..., 0::2] | codes[..., 1::2] << 4
        for t, (u, q) in enumerate(zip(users, pos)):
            block = want[table[u, q // page], layer]
            s = q % page
            block[:, i * n + s * hd // 2:i * n + (s + 1) * hd // 2] = packed[t]
            block[:, 2 * n + i * par + s * hd // 16:2 * n + i * par + (s + 1) * hd // 16] = params[t].reshape(kv, -1).view(np.uint8)
    assert np.array_equal(pool_t.cpu().numpy(), want)
    k_out, v_out = (torch.empty(kv, len(users), hd, dtype=dtype, device="cuda").transpose(0, 1) for _ in range(2))
    kv4.kfl_kv4_read(p, m, layer, int32(users), int32(pos), k_out, v_out)
    for a, b in ((k, k_out), (v, v_out)):
        ref = ora.values(*ora.quantise(a.float().cpu().numpy()))
        assert torch.equal(b.cpu(), torch.from_numpy(ref.astype(np.float32)).to(dtype))
        g = a.double().cpu().numpy().reshape(len(users), kv, -1, 64)
        step = (g.max(-1) - g.min(-1)) / 15
        off = np.abs(ref.reshape(g.shape) - g).max(-1)
        # half a step, the roundings of scale (times 7.5 codes) and centre to fp16
        assert (off <= 0.5 * step + 2.0 ** -11 * (8 * step + np.abs(g).max(-1)) + 2.0 ** -20).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("r", [128, 64, 36, 2])
@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
def test_append_rotates_k(layout, r, dtype):
    hd, kv, page, n = 128, 2, 32, 90
    kv4, pool_t, p, m, _ = cache([n], kv, hd, page)
    plan = kv4.rope_plan(kv4.kfl_rope_table(n, r, THETA), layout)
    odd = torch.empty(n, kv, hd + 1, dtype=dtype, device="cuda")[..., 1:]  # rows off 16 bytes
    k, v, pos = randn((n, kv, hd), dtype, 5), randn((n, kv, hd), dtype, 6), int32(range(n))
    odd.copy_(k)
    user = int32([0] * n)
    k_out, v_out, k2, v2 = (torch.empty(n, kv, hd, device="cuda") for _ in range(4))
    for rows in (k, odd):
        kv4.kfl_kv4_append(p, m, 0, rows, v, user, pos, rope=plan)
        kv4.kfl_kv4_read(p, m, 0, user, pos, k2, v2)
        if rows is k:
            k_out.copy_(k2), v_out.copy_(v2)
    assert torch.equal(k_out, k2) and torch.equal(v_out, v2)
    assert torch.equal(v_out.cpu(), torch.from_numpy(ora.values(*ora.quantise(v.float().cpu().numpy())).astype(np.float32)))
    turned = ora.rotate(k.double().cpu().numpy(), np.arange(n)[:, None] * freqs(r), layout == "interleaved")
    g = turned.reshape(n, kv, -1, 64)
    step = ((g.max(-1) - g.min(-1)) / 15)[..., None]
    off = np.abs(k_out.double().cpu().numpy().reshape(g.shape) - g)
    slack = 2.0 ** -11 * (8 * step + np.abs(g).max(-1)[..., None]) + 2.0 ** -18
    assert (off <= 0.5 * step + slack).all()


def test_groups_that_cannot_be_held_read_as_nan():
    kv4, pool_t, p, m, _ = cache([6], 1, 128, 16)
    k, v = randn((6, 1, 128), FP32, 1), randn((6, 1, 128), FP32, 2)
    k[0, 0, 3], k[1, 0, 64], v[2, 0, 127], v[3, 0, 0] = float("nan"), float("inf"), 32769.0, -float("inf")
    v[4, 0, 5], v[4, 0, 6] = 32768.0, -32768.0
    k[5, 0, :64], k[5, 0, 64:] = 1e-9, -0.0
    pos, user = int32(range(6)), int32([0] * 6)
    kv4.kfl_kv4_append(p, m, 0, k, v, user, pos)
    a, b = torch.empty_like(k), torch.empty_like(v)
    kv4.kfl_kv4_read(p, m, 0, user, pos, a, b)
    bad = [(torch.isnan(x[:, 0, :64]).all(-1).tolist(), torch.isnan(x[:, 0, 64:]).all(-1).tolist(), torch.isnan(x).sum().item())
           for x in (a, b)]
    assert bad[0] == ([True] + [False] * 5, [False, True] + [False] * 4, 128)
    assert bad[1] == ([False] * 3 + [True] + [False] * 2, [False] * 2 + [True] + [False] * 3, 128)
    # the widest group that is held, its step 65536 / 15
    assert (b[4, 0, :64].double().cpu() - v[4, 0, :64].double().cpu()).abs().max() <= 65536 / 30 + 64
    assert (a[5].abs() <= 2.0 ** -24).all()


def test_rows_out_of_range_are_reported_and_not_written():
    kv4, pool_t, p, m, table = cache([20, 5], 2, 64, 16)
    k, v = randn((7, 2, 64), BF16, 1), randn((7, 2, 64), BF16, 2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = pool_t.clone()
    for users, pos, bit in (([0, 0], [-1, 48], kv4.KFL_BAD_POSITION), ([1, 1], [16, 40], kv4.KFL_BAD_POSITION),
                            ([2, -1], [0, 0], kv4.KFL_BAD_USER)):
        status.zero_()
        kv4.kfl_kv4_append(p, m, 0, k[:2], v[:2], int32(users), int32(pos), status=status)
        assert status.item() == bit and torch.equal(pool_t, before)
        out = torch.full((2, 2, 64), 7.0, dtype=BF16, device="cuda")
        status.zero_()
        kv4.kfl_kv4_read(p, m, 0, int32(users), int32(pos), out, out.clone(), status=status)
        assert status.item() == bit and (out == 7).all()
    m.tensors[0][0, 1] = 99
    status.zero_()
    kv4.kfl_kv4_append(p, m, 0, k[:2], v[:2], int32([0, 1]), int32([17, 4]), status=status)
    assert status.item() == kv4.KFL_BAD_PAGE
    assert not torch.equal(pool_t, before)  # the good row is there


def test_calls_without_users_and_without_tokens():
    kv4, pool_t, p, m, table = cache([3, 3, 3], 1, 64, 16)
    k = randn((3, 1, 64), BF16, 4)
    kv4.kfl_kv4_append(p, m, 0, k[:0], k[:0], None, int32([]))
    kv4.kfl_kv4_append(p, m, 0, k, k, None, int32([2, 0, 1]))
    out, out2 = torch.empty_like(k), torch.empty_like(k)
    kv4.kfl_kv4_read(p, m, 0, int32([0, 1, 2]), int32([2, 0, 1]), out, out2)
    ref = torch.from_numpy(ora.values(*ora.quantise(k.float().cpu().numpy())).astype(np.float32)).to(BF16)
    assert torch.equal(out.cpu(), ref) and torch.equal(out2.cpu(), ref)


def test_on_another_stream_and_captured():
    """Calls on a stream of their own, and in a graph that is replayed on changed inputs."""
    kv4, pool_t, p, m, table = cache([40], 2, 128, 16)
    q, k, v = randn((1, 16, 128), BF16, 1), randn((1, 2, 128), BF16, 2), randn((1, 2, 128), BF16, 3)
    pos, user, out, turned = int32([39]), int32([0]), torch.empty_like(q), torch.empty_like(q)
    rows = randn((40, 2, 128), BF16, 7)
    kv4.kfl_kv4_append(p, m, 0, rows, rows, int32([0] * 40), int32(range(40)))
    plan = kv4.rope_plan(kv4.kfl_rope_table(64, 128, THETA))
    ws = kv4.attend_workspace(p, 16, 1, 1)
    torch.cuda.synchronize()

    def step(stream):
        kv4.kfl_rope(plan, q, turned, None, None, pos, cuda_stream=stream)
        kv4.kfl_kv4_append(p, m, 0, k, v, user, pos, rope=plan, cuda_stream=stream)
        kv4.kfl_kv4_attend(p, m, 0, turned, out, ws, users=user, cuda_stream=stream)

    s = torch.cuda.Stream()
    step(s.cuda_stream)
    s.synchronize()
    first = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step(s.cuda_stream)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first)
    q.copy_(randn((1, 16, 128), BF16, 9))
    g.replay()
    torch.cuda.synchronize()
    again = out.clone()
    step(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and not torch.equal(out, first)


@pytest.mark.parametrize("offset", [0.0, 3.0, 1000.0, -20000.0])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
def test_groups_far_from_zero(offset, dtype):
    """The centre's rounding to fp16 is up to many steps there: codes are clamped in some groups, not in others."""
    hd, kv, page, n = 128, 2, 64, 70
    kv4, pool_t, p, m, _ = cache([n], kv, hd, page)
    x = (randn((n, 2 * kv, hd), FP32, seed=11) * torch.logspace(-3, 1, n, device="cuda")[:, None, None] + offset).to(dtype)
    k, v = x[:, :kv], x[:, kv:]
    users, pos = int32(np.zeros(n)), int32(np.arange(n))
    kv4.kfl_kv4_append(p, m, 0, k, v, users, pos)
    out = [torch.empty(n, kv, hd, dtype=FP32, device="cuda") for _ in range(2)]
    kv4.kfl_kv4_read(p, m, 0, users, pos, *out)
    for a, b in zip((k, v), out):
        codes, params = ora.quantise(a.float().cpu().numpy())
        assert torch.equal(b.cpu(), torch.from_numpy(ora.values(codes, params).astype(np.float32)))
    if abs(offset) == 1000.0:
        assert codes.max() == 15 and any((g == 0).sum() > 1 for g in codes.reshape(-1, 64))
