"""New tokens normalised, rotated and appended, against a plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

import plain
from formats_util import K_SCALE, KINDS, V_SCALE, e4m3, make_batch, pools_of, shape_of
from gpu_util import to_bits, to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl

pytestmark = pytest.mark.gpu

EPS = 1e-5


def run(b, pools, starts=None, tokens=None, rotary=None, interleaved=False, norm=(True, True), gap=0, max_ctx=0, in_place=False, scale=1.0, lens=None, eps=EPS):
    """One call on random rows: inputs and outputs as values on the host."""
    hq, hkv, dim, rng = b.hq, b.hkv, b.dim, b.rng
    T = len(b.lens) if starts is None else tokens if tokens is not None else int(starts[-1])
    rotary = dim if rotary is None else rotary
    bound = max_ctx or b.tables.shape[1] * b.block
    width = (hq + 2 * hkv) * dim + gap
    rows = wl.f32_to_bf16_bits(scale * rng.standard_normal((T, width)).astype(np.float32))
    angle = np.arange(bound)[:, None] * 10000.0 ** (-np.arange(0, rotary, 2) / max(rotary, 1))
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    weights = [wl.f32_to_bf16_bits(1 + 0.2 * rng.standard_normal(dim).astype(np.float32)) if n else None for n in norm]
    d = to_dev(rows)
    q_rows = rows[:, :hq * dim]
    q_d, q_stride = d, width
    if in_place:
        q_d, q_stride = to_dev(q_rows), 0
    q_out = q_d if in_place else torch.full((T, hq, dim), 0x7FC1, dtype=torch.int16, device="cuda")
    rope = pkv.make_rope(T, rotary, bound, interleaved=interleaved, norm_eps=eps, q_stride=q_stride, k_stride=width, v_stride=width)
    name = "kv_rope_append" + {"bf16": "", "fp8": "_fp8", "fp4": "_fp4"}[pools.kind]
    scales = (K_SCALE, V_SCALE) if pools.kind == "fp8" else ()
    getattr(pkv, name)(q_d, d[:, hq * dim:], d[:, (hq + hkv) * dim:], *[None if w is None else to_dev(w) for w in weights],
                       to_dev(table) if rotary else None, q_out, pools.k_dev, pools.v_dev, to_dev(b.tables),
                       to_dev(b.lens if lens is None else lens), None if starts is None else to_dev(np.asarray(starts, np.int32)), *scales, rope,
                       shape_of(b, max_ctx))
    torch.cuda.synchronize()
    found = plain.positions(b.lens if lens is None else lens, starts, bound, T)
    x = wl.bf16_bits_to_f64(rows).reshape(T, width)[:, :(hq + 2 * hkv) * dim].reshape(T, -1, dim)
    at = table[[max(p, 0) for _, p in found]]
    w = [None if v is None else wl.bf16_bits_to_f64(v).reshape(dim) for v in weights]
    q, q_size = plain.turn(x[:, :hq], w[0], at, interleaved, eps)
    k, k_size = plain.turn(x[:, hq:hq + hkv], w[1], at, interleaved, eps)
    return dict(found=found, q=q, q_size=q_size, k=k, k_size=k_size, v=x[:, hq + hkv:], q_out=to_bits(q_out).reshape(T, hq, dim), q_rows=q_rows,
                rows=rows)


# fp32: D products in the sum of squares (relative D / 2 * 2^-24 of the root at most), and a handful of roundings
def arithmetic(size, dim):
    return (dim / 2 + 16) * 2.0 ** -24 * size


def check(b, pools, r, faulty=()):
    """q_out, the slots that were written and everything else of the pools."""
    for i, (s, p) in enumerate(r["found"]):
        if s < 0:
            assert (r["q_out"][i] == 0x7FC1).all()
            continue
        plain.within(r["q_out"][i], r["q"][i], 2.0 ** -8 * np.abs(r["q"][i]) + arithmetic(r["q_size"][i], b.dim) + 2.0 ** -130)
    slots = {i: (b.tables[s, p // b.block], p % b.block) for i, (s, p) in enumerate(r["found"]) if s >= 0 and i not in faulty}
    for name, is_v in (("k", False), ("v", True)):
        dev, bits = getattr(pools, name + "_dev"), getattr(pools, name + "_bits")
        got = (to_bits(dev) if pools.kind == "bf16" else dev.cpu().numpy()).reshape(bits.shape)
        new = r["v"] if is_v else r["k"]
        size = np.zeros_like(new) if is_v else arithmetic(r["k_size"], b.dim)
        untouched = np.ones((bits.shape[0], b.block), bool)
        for block, slot in slots.values():
            untouched[block, slot] = False
        if pools.kind == "fp4":
            code_at, scale_at, _ = plain._places(b.dim, is_v)
            for u in range(b.block // 16):
                old = untouched[:, 16 * u:16 * u + 16]
                for at in (code_at, scale_at):
                    g, w = (x[:, :, u][:, :, at] for x in (got, bits))       # [NB, Hkv, 16, D]
                    assert np.array_equal(g.transpose(0, 2, 1, 3)[old], w.transpose(0, 2, 1, 3)[old])
            values = plain.decode(got, b.dim, is_v)
        else:
            assert np.array_equal(got.transpose(0, 2, 1, 3)[untouched], bits.transpose(0, 2, 1, 3)[untouched])
            values = (wl.bf16_bits_to_f64(got).reshape(got.shape) if pools.kind == "bf16"
                      else e4m3(got) * float(np.float32(V_SCALE if is_v else K_SCALE)))
        for i, (block, slot) in slots.items():
            x, y, near = values[block, :, slot], new[i], size[i]
            if pools.kind == "bf16":
                off = 2.0 ** -8 * np.abs(y) + near + 2.0 ** -130
            elif pools.kind == "fp8":   # half a step of e4m3, of its subnormals (2^-9) too; the fp32 division before it
                pool_scale = V_SCALE if is_v else K_SCALE
                y = np.clip(y, -448 * pool_scale, 448 * pool_scale)
                off = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * pool_scale) * (1 + 2.0 ** -20) + 2 * near + 2.0 ** -22 * np.abs(y)
            else:                       # half a step of E2M1 at a scale of at most 2 / 7 of the group's largest
                most = np.repeat(np.abs(y).reshape(b.hkv, -1, 32).max(-1), 32, -1)
                off = np.maximum(np.abs(y) / 4, most / 14) * (1 + 2.0 ** -12) + 2 * near
            assert (np.abs(x - y) <= off).all(), (name, i)
        if is_v and pools.kind == "fp4":    # V comes as it is, so its bytes are the definition's
            want = bits.copy()
            for i, (block, slot) in slots.items():
                plain.put(want, b.dim, [block], [slot], new[i:i + 1], True)
            assert np.array_equal(got, want)


def starts_of(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,block", [(64, 32), (128, 16), (256, 64)])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (5, 1), (12, 12)])
def test_one_token_each(device, kind, dim, block, hq, hkv):
    b = make_batch([1, 16, 17, 300, 33, 0, 512], hq, hkv, dim, block, seed=41, spare=2)
    pools = pools_of(b, kind)
    check(b, pools, run(b, pools))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 0, 3], [0, 0, 200], [16, 17, 15], [130, 64, 1]])
def test_prompts_and_pieces_of_them(device, kind, dim, new):
    past = [0, 21, 70]
    b = make_batch([p + n for p, n in zip(past, new)], 6, 2, dim, 16, seed=sum(new), spare=3)
    pools = pools_of(b, kind)
    check(b, pools, run(b, pools, starts_of(new)))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rotary", [0, 16, 32, 48, 64, 112, 256])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(device, dim, rotary, interleaved):
    if rotary > dim:
        pytest.skip("more than a row")
    b = make_batch([30, 200], 4, 2, dim, 16, seed=rotary)
    pools = pools_of(b, "bf16")
    check(b, pools, run(b, pools, starts_of([30, 5]), rotary=rotary, interleaved=interleaved))


@pytest.mark.parametrize("norm", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("kind", KINDS)
def test_without_weights(device, kind, norm):
    b = make_batch([30, 200], 4, 2, 128, 16, seed=43)
    pools = pools_of(b, kind)
    check(b, pools, run(b, pools, norm=norm))


def test_neither_norm_nor_rotation_is_an_append(device):
    b = make_batch([30, 200, 1], 4, 2, 128, 16, seed=44)
    pools = pools_of(b, "bf16")
    r = run(b, pools, rotary=0, norm=(False, False))
    check(b, pools, r)
    assert np.array_equal(r["q_out"].reshape(3, -1), r["q_rows"])
    k, v = to_dev(pools.k_bits), to_dev(pools.v_bits)
    row = r["rows"][:, 4 * 128:].reshape(3, 4, 128)
    pkv.kv_append(to_dev(row[:, :2].copy()), to_dev(row[:, 2:].copy()), k, v, to_dev(b.tables), to_dev(b.lens), shape_of(b))
    torch.cuda.synchronize()
    assert torch.equal(k, pools.k_dev) and torch.equal(v, pools.v_dev)


@pytest.mark.parametrize("gap", [8, 64])
def test_gaps_and_in_place(device, gap):
    b = make_batch([30, 200, 64], 4, 2, 128, 16, seed=45)
    pools = pools_of(b, "bf16")
    check(b, pools, run(b, pools, starts_of([5, 100, 64]), gap=gap))
    pools = pools_of(b, "bf16")
    check(b, pools, run(b, pools, starts_of([5, 100, 64]), in_place=True, gap=gap))


@pytest.mark.parametrize("kind", KINDS)
def test_padding_and_tokens_without_a_position(device, kind):
    """Rows before the first and behind the last request's, a request with more new tokens than context, an empty one: left as they were."""
    b = make_batch([30, 200, 4, 0, 20], 4, 2, 128, 16, seed=46, spare=4)
    pools = pools_of(b, kind)
    starts = np.array([3, 10, 20, 30, 33, 34], np.int32)      # request 2 has 10 new tokens and a context of 4
    r = run(b, pools, starts, tokens=50)
    assert [i for i, (s, _) in enumerate(r["found"]) if s >= 0] == [*range(3, 20), *range(26, 30), 33]
    check(b, pools, r)
    check(b, pools2 := pools_of(b, kind), run(b, pools2, starts, tokens=12))      # starts that go on behind the rows


@pytest.mark.parametrize("kind", KINDS)
def test_length_bound(device, kind):
    b = make_batch([300, 90, 129], 4, 2, 128, 16, seed=47)
    pools = pools_of(b, kind)
    check(b, pools, run(b, pools, max_ctx=128))
    pools = pools_of(b, kind)
    check(b, pools, run(b, pools, starts_of([10, 90, 3]), max_ctx=128))


@pytest.mark.expects_id_faults
@pytest.mark.parametrize("kind", KINDS)
def test_ids_outside_the_pool(device, id_faults, kind):
    b = make_batch([40, 20, 300], 4, 2, 128, 16, seed=48, spare=1)
    pools = pools_of(b, kind)
    new = [20, 3, 1]
    right = b.tables.copy()
    b.tables[0, 2], b.tables[2, 18] = -1, b.num_blocks           # tokens 32..39 of request 0, the one of request 2
    r = run(b, pools, starts_of(new))
    b.tables = right
    check(b, pools, r, faulty=[*range(12, 20), 23])
    assert int(id_faults.item()) == 9


@pytest.mark.parametrize("seqs", [1, 63, 64, 65, 700, 2048])
def test_requests_are_found(device, seqs):
    """Ragged tokens of many requests, many of them with none."""
    rng = np.random.default_rng(seqs)
    new = rng.integers(0, 3, seqs) * (rng.random(seqs) < 0.6)
    new[rng.integers(0, seqs)] += 2
    b = make_batch(new + rng.integers(0, 20, seqs), 2, 1, 64, 16, seed=seqs)
    pools = pools_of(b, "bf16")
    check(b, pools, run(b, pools, starts_of(new)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,hq,hkv", [(64, 8, 1), (64, 16, 8), (64, 20, 5), (128, 3, 1), (128, 8, 8), (128, 40, 8), (256, 2, 1), (256, 10, 5)])
@pytest.mark.parametrize("ragged", [False, True])
def test_many_tokens(device, kind, dim, hq, hkv, ragged):
    """From 1024 tokens on: rows of several tokens to a workgroup, or several of a token to a lane; with padding, requests with none and ones
    with more tokens than context."""
    rng = np.random.default_rng(dim + hq)
    if ragged:
        new = np.array([0, 700, 1, 0, 0, 333, 40, 2, 60])
        lens = new + np.array([3, 0, 17, 0, 5, 1, -30, 0, 100])       # request 6 has ten tokens of context
        b = make_batch(lens, hq, hkv, dim, 16, seed=52, spare=2)
        pools = pools_of(b, kind)
        check(b, pools, run(b, pools, 2 + starts_of(new), tokens=1151))
    else:
        b = make_batch(rng.integers(0, 40, 1100), hq, hkv, dim, 16, seed=53)
        pools = pools_of(b, kind)
        check(b, pools, run(b, pools))


@pytest.mark.expects_id_faults
def test_many_tokens_with_ids_outside_the_pool(device, id_faults):
    b = make_batch(np.full(40, 30), 3, 1, 64, 16, seed=54, spare=1)
    pools = pools_of(b, "bf16")
    right = b.tables.copy()
    b.tables[7, 1] = b.num_blocks                                # tokens 16..29 of request 7
    r = run(b, pools, starts_of([30] * 40))
    b.tables = right
    check(b, pools, r, faulty=range(7 * 30 + 16, 8 * 30))
    assert int(id_faults.item()) == 14


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** -20, 2.0 ** 40])
def test_small_and_large_rows(device, scale):
    """Squares that leave fp32's range give what fp32 gives, so scales stay within its root; a row of zeros stays zeros."""
    b = make_batch([30, 200, 64], 4, 2, 128, 16, seed=49)
    pools = pools_of(b, "bf16")
    check(b, pools, run(b, pools, scale=scale))
    pools = pools_of(b, "bf16")
    check(b, pools, run(b, pools, scale=0.0))


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_mean_squares_below_the_normal_numbers(device, dim):
    # without an epsilon: rows of about 2^-66, whose mean square of 2^-132 is a subnormal number of fp32.  Squares, their sums and the mean are each
    # off by at most 2^-150, the mean so by less than 3 * 2^-150, which is 2^-16.4 of it, and half of that in the root
    b = make_batch([17, 5, 64, 1], 8, 2, dim, 32, seed=60)
    r = run(b, pools_of(b, "bf16"), scale=2.0 ** -66, eps=0.0)
    assert np.isfinite(r["q"]).all() and np.abs(r["q"]).max() > 1
    plain.within(r["q_out"], r["q"], 2.0 ** -8 * np.abs(r["q"]) + arithmetic(r["q_size"], dim) + 2.0 ** -16 * r["q_size"])


def test_infinities_and_nan_stay_in_their_rows(device):
    b = make_batch([30, 200], 2, 2, 128, 16, seed=50)
    for kind in KINDS:
        pools = pools_of(b, kind)
        rows = wl.normal_bf16(b.rng, (2, 6, 128))
        rows[0, 1, 5], rows[0, 2, 70], rows[1, 5, 3] = wl.BF16_NAN, wl.BF16_NAN, wl.BF16_NAN     # q head 1, k head 0; v head 1
        d = to_dev(rows)
        q_out = torch.empty((2, 2, 128), dtype=torch.int16, device="cuda")
        weight = to_dev(np.full(128, 0x3F80, np.uint16))
        table = to_dev(np.ones((208, 128), np.float32))
        rope = pkv.make_rope(2, 128, 208, q_stride=768, k_stride=768, v_stride=768)
        args = (d, d[:, 2:], d[:, 4:], weight, weight, table, q_out, pools.k_dev, pools.v_dev, to_dev(b.tables), to_dev(b.lens), None)
        {"bf16": lambda: pkv.kv_rope_append(*args, rope, shape_of(b)),
         "fp8": lambda: pkv.kv_rope_append_fp8(*args, K_SCALE, V_SCALE, rope, shape_of(b)),
         "fp4": lambda: pkv.kv_rope_append_fp4(*args, rope, shape_of(b))}[kind]()
        torch.cuda.synchronize()
        nan = np.isnan(wl.bf16_bits_to_f64(to_bits(q_out)).reshape(2, 2, 128))
        assert nan[0, 1].all() and nan.sum() == 128
        for dev, is_v in ((pools.k_dev, False), (pools.v_dev, True)):
            if kind == "bf16":
                x = wl.bf16_bits_to_f64(to_bits(dev)).reshape(b.num_blocks, 2, 16, 128)
            else:
                x = e4m3(dev.cpu().numpy()) if kind == "fp8" else plain.decode(dev.cpu().numpy(), 128, is_v)
            got = [np.isnan(x[b.tables[s, (n - 1) // 16], :, (n - 1) % 16]) for s, n in enumerate(b.lens)]
            want = np.zeros((2, 2, 128), bool)
            if is_v:
                want[1, 1, slice(0, 32) if kind == "fp4" else 3] = True
            else:
                want[0, 0] = True
            assert np.array_equal(np.array(got), want), (kind, is_v)
