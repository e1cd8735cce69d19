"""Rotated appends, windows and 4-bit pools as a serving program runs them: a prompt, decode steps behind it, captured and replayed, pools that
pass 32 bits."""
import numpy as np
import pytest
import torch

import plain
from formats_util import K_SCALE, KINDS, V_SCALE, attend, e4m3, make_batch, pools_of, shape_of
from gpu_util import to_bits, to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl

pytestmark = pytest.mark.gpu

SUFFIX = {"bf16": ("", ""), "fp8": ("_fp8", "_fp8kv"), "fp4": ("_fp4", "_fp4kv")}


class Model:
    """One layer's cache side: projections come in, rows go out."""

    def __init__(self, b, pools, window, sinks):
        self.b, self.pools, self.span = b, pools, (window, sinks)
        self.scales = (K_SCALE, V_SCALE) if pools.kind == "fp8" else ()
        self.append = getattr(pkv, "kv_rope_append" + SUFFIX[pools.kind][0])
        self.attention = getattr(pkv, "paged_decode_attn_window" + SUFFIX[pools.kind][1])
        self.shape = shape_of(b)
        self.bound = b.tables.shape[1] * b.block
        angle = np.arange(self.bound)[:, None] * 10000.0 ** (-np.arange(0, b.dim, 2) / b.dim)
        self.table = to_dev(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32))
        self.norms = [to_dev(wl.f32_to_bf16_bits(1 + 0.2 * b.rng.standard_normal(b.dim).astype(np.float32))) for _ in range(2)]
        self.tables = to_dev(b.tables)
        self.ws = torch.empty(pkv.pkv_attn_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda")

    def put(self, rows, lens, starts, q_out):
        b = self.b
        row = (b.hq + 2 * b.hkv) * b.dim
        rope = pkv.make_rope(rows.shape[0], b.dim, self.bound, q_stride=row, k_stride=row, v_stride=row)
        self.append(rows, rows[:, b.hq * b.dim:], rows[:, (b.hq + b.hkv) * b.dim:], *self.norms, self.table, q_out, self.pools.k_dev,
                    self.pools.v_dev, self.tables, lens, starts, *self.scales, rope, self.shape)

    def step(self, rows, lens, q_out, out):
        self.put(rows, lens, None, q_out)
        self.attention(q_out, self.pools.k_dev, self.pools.v_dev, self.tables, lens, float(self.b.scale), *self.scales, *self.span, out,
                       self.shape, self.ws)


def values(pools, b):
    """The pools' values in 64 bits, as they are on the device."""
    found = []
    for dev, is_v in ((pools.k_dev, False), (pools.v_dev, True)):
        if pools.kind == "bf16":
            x = wl.bf16_bits_to_f64(to_bits(dev))
        elif pools.kind == "fp8":
            x = e4m3(dev.cpu().numpy()) * float(np.float32(V_SCALE if is_v else K_SCALE))
        else:
            x = plain.decode(dev.cpu().numpy(), b.dim, is_v)
        found.append(x.reshape(b.num_blocks, b.hkv, b.block, b.dim))
    return found


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,block", [(64, 32), (128, 16), (256, 16)])
def test_a_prompt_and_decode_steps_eager_and_captured(device, kind, dim, block):
    """Prompts go into the cache in one ragged call, then steps of append and windowed attention, each eager, then the same step as a replay of
    a graph captured once; every step's rows against attention in 64 bits over the pools, and the pools of both ways the same."""
    steps, prompt = 5, np.array([70, 1, 33, 200, 16])
    b = make_batch(prompt + steps, 6, 2, dim, block, seed=61)
    eager, replayed = pools_of(b, kind), None
    for pool in (eager.k_dev, eager.v_dev):
        pool.zero_()
    m = Model(b, eager, 40, 5)
    T, row = int(prompt.sum()), (6 + 4) * dim
    rows = to_dev(wl.normal_bf16(b.rng, (T, row)))
    starts = to_dev(np.concatenate([[0], np.cumsum(prompt)]).astype(np.int32))
    m.put(rows, to_dev(prompt.astype(np.int32)), starts, torch.empty((T, 6, dim), dtype=torch.int16, device="cuda"))
    torch.cuda.synchronize()
    replayed = type(eager)(**{**vars(eager), "k_dev": eager.k_dev.clone(), "v_dev": eager.v_dev.clone()})
    g = Model.__new__(Model)
    g.__dict__.update(m.__dict__)
    g.pools, g.ws = replayed, torch.empty_like(m.ws)

    S = len(prompt)
    rows_s = torch.zeros((S, row), dtype=torch.int16, device="cuda")
    lens_s = to_dev(prompt.astype(np.int32))
    q_s, out_s, q_e, out_e = (torch.zeros((S, 6, dim), dtype=torch.int16, device="cuda") for _ in range(4))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        g.step(rows_s, lens_s, q_s, out_s)
    torch.cuda.synchronize()
    assert torch.equal(eager.k_dev, replayed.k_dev) and torch.equal(eager.v_dev, replayed.v_dev), "a capture executes nothing"
    for i in range(steps):
        lens_s.add_(1)
        rows_s.copy_(to_dev(wl.normal_bf16(b.rng, (S, row))))
        out_s.fill_(0x7FC1), out_e.fill_(0x7FC1)
        m.step(rows_s, lens_s, q_e, out_e)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out_s, out_e) and torch.equal(q_s, q_e), f"step {i}: replay != eager"
        assert torch.equal(eager.k_dev, replayed.k_dev) and torch.equal(eager.v_dev, replayed.v_dev)
        k, v = values(eager, b)
        q = wl.bf16_bits_to_f64(to_bits(q_e)).reshape(S, 6, dim)
        want, off = plain.attention(q, k, v, b.tables, prompt + i + 1, b.scale, 40, 5)
        plain.within(to_bits(out_e), want, off)


@pytest.mark.parametrize("kind", KINDS)
def test_pools_that_pass_32_bits(device, kind):
    """The same blocks at the far end of a pool of more than 4 GiB: the same rows, and the same bytes appended."""
    b = make_batch([300, 75, 1, 900], 8, 2, 128, 16, seed=62)
    pools = pools_of(b, kind)
    size = pools.k_dev.numel() * pools.k_dev.element_size() // b.num_blocks
    far = (5 << 30) // size
    big = [torch.empty((far + b.num_blocks) * size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ids = to_dev(np.arange(far, far + b.num_blocks, dtype=np.int32))
    for src, dst in ((pools.k_dev, big[0]), (pools.v_dev, big[1])):
        pkv.kv_blocks_scatter(src, dst, ids, b.num_blocks, size, far + b.num_blocks)
    small = Model(b, pools, 200, 3)
    rows = to_dev(wl.normal_bf16(b.rng, (4, 12 * 128)))
    lens = to_dev(b.lens)
    q, out = (torch.zeros((4, 8, 128), dtype=torch.int16, device="cuda") for _ in range(2))
    small.step(rows, lens, q, out)
    torch.cuda.synchronize()
    tables, n = b.tables, b.num_blocks
    b.tables, b.num_blocks = np.where(tables >= 0, tables + far, -1).astype(np.int32), far + n
    large = Model.__new__(Model)
    large.__dict__.update(small.__dict__)
    large.pools = type(pools)(kind=kind, k_dev=big[0], v_dev=big[1])
    large.tables, large.shape = to_dev(b.tables), shape_of(b)
    q2, out2 = torch.zeros_like(q), torch.zeros_like(out)
    large.step(rows, lens, q2, out2)
    torch.cuda.synchronize()
    assert torch.equal(q, q2) and torch.equal(out, out2)
    for src, dst in ((pools.k_dev, big[0]), (pools.v_dev, big[1])):
        assert torch.equal(src.view(-1).view(torch.uint8), dst[far * size:])
    whole = attend(b, large.pools), None
    b.tables, b.num_blocks = tables, n
    assert np.array_equal(whole[0], attend(b, pools))


@pytest.mark.parametrize("tokens", [3, 1100])
def test_rows_that_pass_32_bits(device, tokens):
    """Rows so far apart that their offsets pass 32 bits."""
    stride = (1 << 32) // tokens // 8 * 8 + 1024
    b = make_batch(np.full(tokens, 2), 2, 1, 128, 16, seed=63)
    near, far = pools_of(b, "bf16"), None
    far = type(near)(kind="bf16", k_dev=near.k_dev.clone(), v_dev=near.v_dev.clone())
    rows = to_dev(wl.normal_bf16(b.rng, (tokens, 4 * 128)))
    wide = torch.empty(tokens * stride, dtype=torch.int16, device="cuda")
    wide.as_strided((tokens, 512), (stride, 1)).copy_(rows)
    table = to_dev(np.ones((16, 128), np.float32))
    outs = []
    for buf, s, p in ((rows.view(-1), 512, near), (wide, stride, far)):
        q_out = torch.zeros((tokens, 2, 128), dtype=torch.int16, device="cuda")
        pkv.kv_rope_append(buf, buf[256:], buf[384:], None, None, table, q_out, p.k_dev, p.v_dev, to_dev(b.tables), to_dev(b.lens), None,
                           pkv.make_rope(tokens, 128, 16, q_stride=s, k_stride=s, v_stride=s), shape_of(b))
        outs.append(q_out)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and torch.equal(near.k_dev, far.k_dev) and torch.equal(near.v_dev, far.v_dev)


def test_calls_on_a_side_stream(device):
    """A prompt's append and the attention behind it, in order on a stream that is not the current one."""
    b = make_batch([500, 90, 30], 4, 2, 128, 16, seed=64)
    pools = pools_of(b, "fp4")
    m = Model(b, pools, 100, 4)
    rows, lens = to_dev(wl.normal_bf16(b.rng, (3, 8 * 128))), to_dev(b.lens)
    q, out, q2, out2 = (torch.zeros((3, 4, 128), dtype=torch.int16, device="cuda") for _ in range(4))
    m.step(rows, lens, q, out)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m.step(rows, lens, q2, out2)
    side.synchronize()
    assert torch.equal(q, q2) and torch.equal(out, out2)
