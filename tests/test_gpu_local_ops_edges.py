"""Cases of the local-step operators that once went wrong or were never reached, against 64-bit values."""
import math

import pytest
import torch

from paper_1909_09010_b200 import binding

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ops():
    return binding.local_ops(0)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rnd(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_out", [8, 33, 1024, 40_000])
@pytest.mark.parametrize("rows", [1, 63, 64, 255, 300, 700, 4096])
def test_bias_gradient_of_every_cluster_size(ops, dtype, rows, n_out):
    """Column sums by clusters of 1, 2, 4 and 8 CTAs, by pieces and element by element, many times over."""
    dz = rnd(gen(rows + n_out), (rows, n_out), dtype)
    x = torch.ones((rows, 8), dtype=dtype, device="cuda")
    ref, size = dz.double().sum(0), dz.double().abs().sum(0)
    first = ops.linear_backward_weight(dz, x, grad_dtype=F)[1]
    # an fp32 sum of `rows` terms in any order, each addition off by half a unit of a partial sum
    assert bool(((first.double() - ref).abs() <= rows * 2.0 ** -24 * size).all())
    for _ in range(20):
        assert torch.equal(ops.linear_backward_weight(dz, x, grad_dtype=F)[1], first)
    assert ops.device_status() == 0


def test_clip_on_another_stream_right_after_new_tensors():
    """The table of the tensors is on the GPU when create and set_tensors return, whatever stream comes next
    and however much the default stream still has to do."""
    g = gen(11)
    sets = [[(rnd(g, s, F), torch.zeros(s, device="cuda"), i % 2) for i, s in enumerate(shapes)]
            for shapes in ([(50_000,), (7, 9)], [(3,), (1000, 40), (123,)], [(9001,), (5,), (64, 64), (2,)])]
    refs = [[math.sqrt(sum(float((t.double() ** 2).sum()) for t, _, k in e if k == j)) for j in range(2)] for e in sets]
    norms = torch.zeros(2, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for turn in range(30):
        i = turn % 3
        torch.cuda._sleep(1_000_000)                       # half a millisecond of work on the default stream
        if turn % 10 == 0:
            clip = binding.GradClip(sets[i], groups=2)
        else:
            clip.set_tensors(sets[i])
        clip.clip(1.0, norms_out=norms, stream=side)
        side.synchronize()
        assert all(abs(float(n) - r) <= 2.0 ** -22 * r for n, r in zip(norms, refs[i]))
        for t, out, k in sets[i]:
            assert torch.allclose(out.double(), t.double() / max(1.0, refs[i][k]), rtol=2.0 ** -20, atol=0)
        for _, out, _ in sets[i]:
            out.zero_()
        torch.cuda.synchronize()
    assert clip.device_status() == 0


def test_new_tensors_keep_a_status_nobody_has_read():
    x, out = torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda")
    clip = binding.GradClip([(x, out, 0)])
    assert clip.device_status() == binding.GBMUF_OK
    clip.selftest_wait_timeout()                           # two seconds, then the word is set
    clip.set_tensors([(x[:500], None, 0), (x[500:], out[500:], 0)])
    assert clip.device_status() == binding.ERR_TIMEOUT and clip.device_status() == binding.GBMUF_OK
    assert abs(float(clip.clip(1.0)[0]) - 1000 ** 0.5) < 1e-5


@pytest.mark.parametrize("more", [False, True])
def test_graph_keeps_the_tensors_it_was_recorded_with(more):
    """New tensors, fewer or many more, neither change nor invalidate what a graph does."""
    g = gen(13)
    first = [(rnd(g, s, F), torch.zeros(s, device="cuda"), 0) for s in [(300_000,), (41, 7)]]
    shapes = [(777,)] * 500 if more else [(5,)]
    second = [(rnd(g, s, F), torch.zeros(s, device="cuda"), 0) for s in shapes]
    length = lambda e: math.sqrt(sum(float((t.double() ** 2).sum()) for t, _, _ in e))              # noqa: E731
    clip = binding.GradClip(first)
    norms, graph = torch.zeros(1, device="cuda"), torch.cuda.CUDAGraph()
    clip.clip(0.5)
    with torch.cuda.graph(graph):
        clip.clip(0.5, norms_out=norms)
    want = [out.clone() for _, out, _ in first]
    clip.set_tensors(second)
    for _ in range(2):
        for _, out, _ in first:
            out.zero_()
        graph.replay()
        assert abs(float(clip.clip(0.5)[0]) - length(second)) <= 2.0 ** -22 * length(second)
        assert abs(float(norms[0]) - length(first)) <= 2.0 ** -22 * length(first)
        assert all(torch.equal(out, w) for (_, out, _), w in zip(first, want))
        clip.set_tensors(second[:1])
        clip.set_tensors(second)
    torch.cuda.synchronize()
    del graph


def test_calls_on_a_side_stream_leave_the_memory_of_pending_work_alone(ops):
    """Blocks that the current stream's pending work still reads are free for that stream's next
    allocation, not for a call that runs on another stream at once."""
    g = gen(17)
    x, w, b = rnd(g, (300, 131), F), rnd(g, (77, 131), F), rnd(g, (77,), F)
    xb, wb = rnd(g, (640, 512), BF), rnd(g, (1024, 512), BF)
    logits, t = rnd(g, (60, 5003), BF, 3.0), torch.randint(0, 5003, (60,), generator=g, device="cuda")
    dz, clip = rnd(g, (60, 77), F), binding.GradClip([(x, None, 0)], groups=65_536)
    work = [lambda s: ops.linear_forward(x, w, bias=b, activation="gelu", keep_z=True, stream=s),
            lambda s: ops.linear_forward(xb, wb, stream=s),
            lambda s: ops.linear_backward_input(dz, w, stream=s),
            lambda s: ops.linear_backward_weight(xb, xb, grad_dtype=F, stream=s),
            lambda s: ops.cross_entropy(logits, t, stream=s), lambda s: ops.activation_backward(xb, xb, "tanh", stream=s),
            lambda s: clip.norms(stream=s)]
    flat = lambda r: r if isinstance(r, tuple) else (r,)                            # noqa: E731
    refs = [flat(f(None)) for f in work]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for f, ref in zip(work, refs):
        # a block of the size of each result and of typical workspaces, read late by the current stream
        blocks = [torch.full((n,), 3.0, device="cuda") for n in {(r.numel() * r.element_size() + 3) // 4 for r in ref} |
                  {80_000, 120_000, 170_000, 250_000}]
        late = [torch.empty_like(v) for v in blocks]
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)                      # ten milliseconds
        for v, out in zip(blocks, late):
            out.copy_(v)
        blocks.clear()
        del v
        got = flat(f(side.cuda_stream if f is work[0] else side))
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, ref))
        torch.cuda.synchronize()
        assert all(bool((out == 3.0).all()) for out in late), "memory of pending work was overwritten"
        del got
    assert ops.device_status() == 0


def test_calls_on_side_streams_in_turn(ops):
    """fp32 products (with a workspace each) on the current stream and on two others, nothing between them."""
    g = gen(19)
    jobs = [(rnd(g, (700 + i, 515), F), rnd(g, (333, 515), F)) for i in range(6)]
    refs = [ops.linear_forward(x, w) for x, w in jobs]
    streams = [None, torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [ops.linear_forward(x, w, stream=streams[i % 3]) for i, (x, w) in enumerate(jobs)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, refs))


@pytest.mark.parametrize("dtype", [BF, F])
def test_clip_with_infinite_bound_copies(dtype):
    """max_norm = inf: nothing is longer than that, so outputs are the gradients."""
    g = gen(3)
    grads = [rnd(g, s, dtype) for s in [(70_001,), (33, 5), (9,)]]
    outs = [torch.full_like(t, 7.0, dtype=F) for t in grads]
    bad, zeroed = rnd(g, (50,), dtype), torch.ones(50, device="cuda")
    bad[3] = math.inf
    clip = binding.GradClip([(t, o, 0) for t, o in zip(grads, outs)] + [(bad, zeroed, 1)], groups=2)
    norms = clip.clip(math.inf)
    ref = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    assert abs(float(norms[0]) - ref) <= 2.0 ** -22 * ref and float(norms[1]) == math.inf
    assert all(torch.equal(o, t.float()) for t, o in zip(grads, outs)) and not bool(zeroed.any())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows", [4, 16, 17, 200])
def test_infinite_operands_give_what_the_plain_product_gives(ops, dtype, rows):
    """An infinity times a finite value is an infinity of the product's sign, infinities of both signs in
    one sum or one times zero are NaN -- whichever kernel takes the call."""
    g = gen(rows)
    x, w = rnd(g, (rows, 320), dtype), rnd(g, (160, 320), dtype, 0.1)
    dz = rnd(g, (rows, 160), dtype)
    x[0, 7], x[1, 300] = math.inf, -math.inf
    x[2, 5] = x[2, 11] = math.inf
    x[3, 0] = math.nan
    w[9, 7], w[11, 300] = 0.0, -math.inf
    w[13, 17] = w[14, 17] = math.inf
    dz[0, 3], dz[1, 13] = -math.inf, math.inf
    wide = lambda *t: [v.double().cpu() for v in t]                                 # noqa: E731
    xd, wd, dd = wide(x, w, dz)
    for got, ref in [(ops.linear_forward(x, w), xd @ wd.t()), (ops.linear_backward_input(dz, w), dd @ wd),
                     (ops.linear_backward_weight(dz, x, want_bias=False), dd.t() @ xd)]:
        got = got.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(torch.isposinf(got), torch.isposinf(ref)) and torch.equal(torch.isneginf(got), torch.isneginf(ref))
        assert bool(torch.isinf(ref).any())


@pytest.mark.parametrize("act,far", [("gelu", 12.0), ("sigmoid", 80.0), ("tanh", 40.0)])
def test_slopes_keep_their_digits_in_the_tails(ops, act, far):
    """Relative errors, where the slope itself is tiny: it is not formed as a difference of numbers near 1."""
    z = torch.linspace(-far, far, 30_000, device="cuda").view(-1, 16)
    zd = z.double()
    if act == "gelu":
        tail, bell = torch.special.erfc(-zd / 2 ** 0.5) / 2, zd * torch.exp(-zd * zd / 2) / math.sqrt(2 * math.pi)
        # both parts are exponentials of z^2 / 2, which is rounded: z^2 2^-24 twice over; 2^-20 for the rest
        ref, tol = tail + bell, (zd * zd * 2.0 ** -23 + 2.0 ** -20) * (tail + bell.abs())
    else:
        e = torch.exp(-zd.abs() * (1 if act == "sigmoid" else 2))
        ref = e / (1 + e) ** 2 * (1 if act == "sigmoid" else 4)
        tol = 2.0 ** -20 * ref               # an exponential of 2 units and five roundings
    eye = torch.eye(16, device="cuda")
    for got in (ops.activation_backward(torch.ones_like(z), z, act),
                ops.linear_backward_input(torch.ones_like(z), eye, z_prev=z, activation=act)):
        err = (got.double() - ref).abs()
        assert bool((err <= tol).all()), float((err / ref.abs()).max())
    if act != "gelu":                        # bf16: single instructions, off by 2^-22 and by |z| 2^-23; then one rounding
        zb = z.to(BF)
        e = torch.exp(-zb.double().abs() * (1 if act == "sigmoid" else 2))
        ref = e / (1 + e) ** 2 * (1 if act == "sigmoid" else 4)
        got = ops.activation_backward(torch.ones_like(zb), zb, act).double()
        assert bool(((got - ref).abs() <= 2.0 ** -8 * ref).all())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab", [1000, 30_001, 267_735])
def test_loss_of_rows_with_a_large_common_offset(ops, dtype, vocab):
    """The loss does not see what all logits of a row have in common, up to rows of the lowest value."""
    x = torch.round(rnd(gen(vocab), (4, vocab), F, 2.0) * 4) / 4            # exact in fp32 beside the offsets below
    offset = torch.tensor([0.0, 2.0 ** 20, -2.0 ** 21, 0.0], device="cuda")[:, None]
    x = x + offset if dtype is F else x.to(dtype)
    x[3, :] = torch.finfo(dtype).min
    t = torch.tensor([1, vocab - 1, vocab // 2, 0], device="cuda")
    loss, lse, d = ops.cross_entropy(x, t, scale=0.5)
    ref = 0.5 * (torch.logsumexp(x.double(), 1) - x.double()[torch.arange(4), t])
    ref[3] = 0.5 * math.log(vocab)                                           # lost in 64 bits as well
    # a sum in chains of at most 300 terms is off by 2^-15 of itself, its log by that; then sums of numbers below 64
    assert bool(((loss.double() - ref).abs() <= 0.5 * (2.0 ** -15 + 64 * 2.0 ** -22)).all()), loss - ref


@pytest.mark.parametrize("dtype", [BF, F])
def test_norms_of_equal_elements(dtype):
    """Every fp32 rounding of a sum of equal squares goes the same way: five of them (six for bf16) and
    the norm's own stay within 2^-22, at any length and across the range."""
    values = [1.0, 1.1, 1.0 + 2.0 ** -7, 1.7, 0.3, 1.9921875, 1e-3, 3e-12, 1e-13, 1e-20, 1e18, 3e19, 1e25, 1e-30]
    grads = [torch.full((n,), v, device="cuda").to(dtype) for v in values for n in (1, 3, 33, 4096, 100_003)]
    norms = binding.GradClip([(t, None, i) for i, t in enumerate(grads)], groups=len(grads)).norms().cpu()
    for t, n in zip(grads, norms):
        ref = math.sqrt(t.numel()) * float(t[0].double())
        assert abs(float(n) - ref) <= 2.0 ** -22 * ref, (t.numel(), float(t[0]), float(n), ref)


def test_adagrad_with_an_infinite_clip_norm_does_not_clip():
    states = []
    for clip_norm in (math.inf, 0.0):
        theta, accum = torch.ones((2, 4096), device="cuda"), torch.full((2, 4096), 0.1, device="cuda")
        omega, delta = torch.zeros_like(theta), torch.zeros_like(theta)
        ctx = binding.Gbmuf(theta, omega, delta, K=2, N=4096, ld=4096, p=0, q=0, eta=0.9, zeta=1.0)
        ctx.set_partition([0, 1000, 4096])
        grad = rnd(gen(31), (2, 4096), F, 5.0)
        ctx.local_adagrad(grad, accum, 0.1, eps=1e-8, clip_norm=clip_norm, clip_mask=[1, 0])
        torch.cuda.synchronize()
        ctx.destroy()
        states.append((theta, accum))
    assert bool(torch.isfinite(states[0][0]).all())
    assert all(torch.equal(p, q) for p, q in zip(*states))


def test_stream_handles(ops):
    """Streams given as torch streams, as their handles, and as the two names of the default stream."""
    g = gen(37)
    x, w = rnd(g, (40, 131), F), rnd(g, (77, 131), F)
    ref = ops.linear_forward(x, w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream, torch.cuda.default_stream(), 0, 1):
        got = ops.linear_forward(x, w, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, ref)
    with torch.cuda.stream(side):
        got = ops.linear_forward(x, w, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got, ref)


def test_round_and_linear_layers_in_turn(ops):
    """Synchronisation rounds with their tile in tensor memory and tensor-core products, each launched
    while the one before still runs: same results as one at a time."""
    g = gen(41)
    K, N = 4, 200_000
    x, w = rnd(g, (512, 256), BF), rnd(g, (1024, 256), BF)
    big, v = rnd(g, (4096, 512), BF), rnd(g, (2048, 512), BF)
    refs = ops.linear_forward(x, w), ops.linear_forward(big, v)
    start = rnd(g, (K, N), F)
    outcomes = []
    for wait in (True, False):
        theta = start.clone()
        omega, delta = start.clone(), torch.zeros_like(start)
        ctx = binding.Gbmuf(theta, omega, delta, K=K, N=N, ld=N, p=1, q=1, eta=0.5, zeta=1.0, seed=3)
        ctx.set_partition([0, 70_001, N])
        torch.cuda.synchronize()
        got = []
        for t in range(1, 9):
            ctx.sync_round(t)
            if wait:
                torch.cuda.synchronize()
            got += [ops.linear_forward(x, w), ops.linear_forward(big, v)]
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert ctx.device_status() == 0
        ctx.destroy()
        assert all(torch.equal(a, refs[i % 2]) for i, a in enumerate(got))
        outcomes.append(torch.stack([theta, omega, delta]))
    assert torch.equal(*outcomes) and not torch.equal(outcomes[0][0], start)
