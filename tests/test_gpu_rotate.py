"""Norms and rotation on the GPU against their definition in 64 bits (oracle/rotate_torch.py)."""
import math

import pytest
import torch

from oracle import rotate_torch as ref
from paper_2309_12307_b200 import binding as s2a
from paper_2309_12307_b200.autograd import s2_rotate

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn

# Results are rounded to bf16 once: half a step, 2^-8 of the value.  Before that: sums of d squares as 16 terms and then a tree of 3, a reciprocal root and
# products, each 2^-24 or 2^-23 of what it gives, together below 2^-18 of the pair's magnitudes; angles off by 2^-23 or less and sines by 2^-22.
HALF, CHAIN = 2.0**-8, 2.0**-18


def radians(r, base=10000.0, scale=1.0):
    return [scale * base ** (-2 * i / r) for i in range(r // 2)]


def near(got, want, size):
    got = got.double().cpu()
    number = ~torch.isnan(want)  # (a row with an infinity has none where it is, and where that turns to)
    assert torch.equal(~torch.isnan(got), number)
    got, want, size = got[number], want[number], size[number]
    off = (got - want).abs()
    allowed = HALF * (want.abs() + CHAIN * size) + CHAIN * size
    assert (off <= allowed).all(), float((off / allowed).max())


def numbers(g, *shape, by=1.0):
    return (torch.randn(shape, generator=g) * by).to(BF16)


class Job:
    def __init__(self, T, H, Hkv, d, r=None, norm=None, weights=BF16, interleaved=False, packed=False, first=0, scale=1.0, seed=0, by=1.0, eps=1e-5):
        g = torch.Generator().manual_seed(seed)
        self.r = d if r is None else r
        self.radians = radians(self.r, scale=scale)
        self.turns = s2a.rotary_turns(self.r, scale=scale)
        self.interleaved = interleaved
        all_three = numbers(g, T, H + 2 * Hkv, d, by=by)
        self.q, self.k = all_three[:, :H], all_three[:, H:H + Hkv]
        on = all_three.cuda()
        self.on_q, self.on_k = on[:, :H], on[:, H:H + Hkv]
        if not packed:
            self.on_q, self.on_k = self.on_q.contiguous(), self.on_k.contiguous()
        self.positions = torch.arange(first, first + T, dtype=torch.int32)
        self.eps = eps if norm else None
        self.qw = self.kw = None
        if norm == "weights":
            self.qw, self.kw = ((1 + 0.3 * torch.randn(d, generator=g)).to(weights) for _ in range(2))
        self.dq_out, self.dk_out = numbers(g, T, H, d), numbers(g, T, Hkv, d)
        self.d = d

    @property
    def how(self):
        return dict(positions=self.positions.cuda(), q_weight=None if self.qw is None else self.qw.cuda(), k_weight=None if self.kw is None else self.kw.cuda(),
                    eps=self.eps, interleaved=self.interleaved)

    def size(self, x):
        return ref.reach(x, self.d, self.r // 2, self.interleaved)

    def check_forward(self):
        got = s2a.s2a_rotate(self.on_q, self.on_k, self.turns, **self.how)
        for y, x, w in zip(got, (self.q, self.k), (self.qw, self.kw)):
            want = ref.rotate(x, self.positions, self.radians, self.interleaved, w, self.eps)
            before = ref.rotate(x, self.positions, [], self.interleaved, w, self.eps)
            near(y, want, self.size(before))
        assert s2a.device_status() == (0, 0)
        return got

    def check_backward(self):
        got = s2a.s2a_rotate_bwd(self.on_q, self.on_k, self.dq_out.cuda(), self.dk_out.cuda(), self.turns, **self.how)
        for dx, dw, x, dy, w in zip(got[:2], got[2:], (self.q, self.k), (self.dq_out, self.dk_out), (self.qw, self.kw)):
            want, want_w = ref.rotate_bwd(x, dy, self.positions, self.radians, self.interleaved, w, self.eps)
            size = self.size(dy)  # of the pairs that turned back
            if self.eps is not None:
                s = 1 / (x.double().square().mean(-1, keepdim=True) + self.eps).sqrt()
                n = x.double() * s
                weighted = size * (1 if w is None else w.double().abs())
                size_x = s * (weighted + n.abs() * (weighted * n.abs()).mean(-1, keepdim=True))
                near(dx, want, 2 * size_x)
            else:
                near(dx, want, size)
            assert (dw is None) == (w is None)
            if w is not None:
                terms = (size * n.abs()).sum((0, 1))
                # besides the terms' own errors the sum's: at most 64 rows of a lane, 64 lanes and blocks' sums one after the other, 2^-24 each
                off = (dw.double().cpu() - want_w).abs()
                allowed = (2 * CHAIN + (64 + 64 + 1000) * 2.0**-24) * terms
                assert dw.dtype == F32 and (off <= allowed).all(), float((off / allowed).max())
        assert s2a.device_status() == (0, 0)
        return got


SHAPES = [(5, 300, 260, 64), (3, 129, 128, 128), (1, 1, 1, 64), (1, 32, 8, 128), (2, 3, 5, 64), (33, 4, 2, 128), (129, 9, 1, 64), (701, 16, 4, 64), (1000, 40, 40, 128), (257, 64, 8, 128)]


@pytest.mark.parametrize("T,H,Hkv,d", SHAPES)
@pytest.mark.parametrize("norm", [None, "plain", "weights"])
def test_forward_and_gradients(T, H, Hkv, d, norm):
    job = Job(T, H, Hkv, d, norm=norm, seed=T, first=T)
    job.check_forward()
    job.check_backward()


@pytest.mark.parametrize("d,r", [(64, 0), (64, 16), (64, 32), (64, 48), (128, 16), (128, 64), (128, 112), (128, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [None, "weights"])
def test_some_of_the_values_and_either_pairing(d, r, interleaved, norm):
    job = Job(37, 6, 3, d, r=r, interleaved=interleaved, norm=norm, packed=True, weights=F32, first=5)
    q, k = job.check_forward()
    job.check_backward()
    if norm is None:  # what is not rotated is not touched
        assert torch.equal(q[..., r:].cpu(), job.q[..., r:]) and torch.equal(k[..., r:].cpu(), job.k[..., r:])


@pytest.mark.parametrize("first", [99_990, 2**31 - 40, -(2**31), -17])
@pytest.mark.parametrize("scale", [1.0, 0.125])
def test_angles_of_far_positions(first, scale):
    job = Job(37, 2, 1, 128, first=first, scale=scale)
    # (the definition itself, in 64 bits: an angle of 2^31 radians is off by 2^-22)
    job.check_forward()
    job.check_backward()


def test_frequencies_in_turns():
    turns = s2a.rotary_turns(128, base=500000.0, scale=0.25, device="cpu")
    want = [0.25 * 500000.0 ** (-2 * i / 128) / (2 * math.pi) for i in range(64)]
    # a whole number of 2^-64 is off by half of that, the quotient (and int / 2**64) by 2^-53 of its value
    assert turns.dtype == torch.int64 and all(abs(int(t) / 2**64 - w) <= 2.0**-65 + 2 * 2.0**-53 * w for t, w in zip(turns, want))
    # more than half a turn a position, and backwards
    assert [int(t) for t in s2a.turns_of([1.5 * math.pi, -0.5 * math.pi], device="cpu")] == [-(2**62)] * 2
    assert s2a.rotary_turns(0).shape == (0,)


def test_positions_by_default_and_for_the_last_dimension():
    g = torch.Generator().manual_seed(1)
    q, k = numbers(g, 3, 50, 4, 64).cuda(), numbers(g, 3, 50, 2, 64).cuda()
    turns = s2a.rotary_turns(64)
    count = torch.arange(50, dtype=torch.int32, device="cuda")
    want = s2a.s2a_rotate(q, k, turns, positions=count.expand(3, 50).contiguous())
    for positions in (None, count):
        got = s2a.s2a_rotate(q, k, turns, positions=positions)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    flat = s2a.s2a_rotate(q.view(150, 4, 64), k.view(150, 2, 64), turns, positions=count.repeat(3))
    assert torch.equal(flat[0].view_as(q), want[0])


def test_into_given_tensors_and_in_place():
    job = Job(65, 8, 2, 128, norm="weights", packed=True)
    want = s2a.s2a_rotate(job.on_q, job.on_k, job.turns, **job.how)
    packed = torch.full((65, 12, 128), 7.0, dtype=BF16, device="cuda")
    got = s2a.s2a_rotate(job.on_q, job.on_k, job.turns, q_out=packed[:, :8], k_out=packed[:, 8:10], **job.how)
    assert got[0].data_ptr() == packed.data_ptr() and torch.equal(packed[:, :8], want[0]) and torch.equal(packed[:, 8:10], want[1]) and (packed[:, 10:] == 7).all()
    s2a.s2a_rotate(job.on_q, job.on_k, job.turns, q_out=job.on_q, k_out=job.on_k, **job.how)
    assert torch.equal(job.on_q, want[0]) and torch.equal(job.on_k, want[1])


@pytest.mark.parametrize("by,eps", [(2.0**100, 1e-5), (2.0**126, 1e-5), (2.0**-100, 0.0), (2.0**-126, 0.0), (2.0**-100, 1e-5), (2.0**-60, 1e-30), (2.0**60, 1e30), (1.0, 3e38)])
def test_rows_whose_squares_leave_the_range(by, eps):
    job = Job(9, 3, 1, 64, norm="weights", by=by, eps=eps)
    job.q[2], job.on_q[2] = 0, 0
    if eps == 0.0:
        job.q[2, :, 0], job.on_q[2, :, 0] = 1.0, 1.0
    job.check_forward()


@pytest.mark.parametrize("by,eps,power", [(2.0**125, 1e-5, 60), (2.0**125, 0.0, 110), (2.0**100, 1e-5, 0), (2.0**60, 1e30, 0), (1.0, 3e38, 40), (2.0**-60, 1e-30, 0), (2.0**-100, 1e-5, 0),
                                          (2.0**-100, 0.0, -20), (2.0**-125, 0.0, -20), (2.0**-131, 0.0, -60), (2.0**-133, 0.0, -100)])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_rows_whose_squares_leave_the_range(by, eps, power, d):
    job = Job(9, 3, 1, d, norm="weights", by=by, eps=eps)
    for t in (job.q, job.on_q, job.k, job.on_k):
        t[..., 0] = by  # (no row of zeros)
    job.dq_out *= 2.0**power
    job.dk_out *= 2.0**power
    job.check_backward()


def test_what_is_not_finite_stays_in_its_row():
    job = Job(40, 4, 2, 64, norm="plain")
    clean = s2a.s2a_rotate(job.on_q, job.on_k, job.turns, **job.how)
    job.on_q[3, 1, 5], job.on_q[7, 2, 63], job.on_k[9, 0, 0] = math.nan, math.inf, -math.inf
    q, k = s2a.s2a_rotate(job.on_q, job.on_k, job.turns, **job.how)
    assert torch.isnan(q[3, 1]).all() and torch.isnan(q[7, 2]).any() and torch.isnan(k[9, 0]).any()
    for y, x, rows in ((q, clean[0], ((3, 1), (7, 2))), (k, clean[1], ((9, 0),))):
        other = torch.ones(x.shape[:2], dtype=torch.bool, device="cuda")
        for r in rows:
            other[r] = False
        assert torch.equal(y[other], x[other])


def test_the_same_twice_and_on_another_stream():
    job = Job(513, 16, 4, 128, norm="weights")
    args = (job.on_q, job.on_k, job.dq_out.cuda(), job.dk_out.cuda(), job.turns)
    how = job.how
    first = s2a.s2a_rotate_bwd(*args, **how)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    again = s2a.s2a_rotate_bwd(*args, **how, stream=stream)
    stream.synchronize()
    with torch.cuda.stream(stream):
        third = s2a.s2a_rotate_bwd(*args, **how)
    stream.synchronize()
    for other in (again, third):
        assert all(torch.equal(a, b) for a, b in zip(first, other))


def test_captured_calls_follow_their_inputs():
    job = Job(64, 8, 8, 64, norm="weights")
    how, q, k, dq, dk = job.how, job.on_q, job.on_k, job.dq_out.cuda(), job.dk_out.cuda()
    s2a.s2a_rotate_bwd(q, k, dq, dk, job.turns, **how)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s2a.s2a_rotate(q, k, job.turns, **how)
        grads = s2a.s2a_rotate_bwd(q, k, dq, dk, job.turns, **how)
    for step in range(2):
        how["positions"] += 1000
        q.mul_(-1.5)
        graph.replay()
        want = s2a.s2a_rotate(q, k, job.turns, **how) + s2a.s2a_rotate_bwd(q, k, dq, dk, job.turns, **how)
        assert all(torch.equal(a, b) for a, b in zip(out + grads, want))


# ---------------------------------------------------------------------------------------------- into the cache
@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("H,Hkv,d,page,norm", [(1, 1, 64, 16, None), (8, 2, 128, 64, "weights"), (40, 40, 128, 32, None), (5, 5, 64, 256, "plain"), (64, 8, 128, 128, "weights")])
@pytest.mark.parametrize("given", [False, True])
def test_into_the_cache_as_by_two_calls(dtype, H, Hkv, d, page, norm, given):
    from test_gpu_paged import Job as CacheJob

    def cache_job():
        return CacheJob([(3, 50), (0, 0), (1, 1), (0, 17), (33, 33), (page, 3 * page), (1, page + 1)], Hkv=Hkv, H=H, d=d, page=page, dtype=dtype, before=2, after=3)

    one, two = cache_job(), cache_job()
    job = Job(one.T, H, Hkv, d, norm=norm, packed=True)
    v = torch.randn(one.T, Hkv, d, generator=torch.Generator().manual_seed(9)).to(BF16).cuda()
    place = torch.zeros(one.T, dtype=torch.int32)
    for b, (n, length) in enumerate(one.sizes):
        start = int(one.starts[b])
        place[start:start + n] = torch.arange(length - n, length)
    how = job.how
    how["positions"] = place.cuda() * 3 + 1000 if given else place.cuda()
    q_want, k_want = s2a.s2a_rotate(job.on_q, job.on_k, job.turns, **how)
    s2a.s2a_cache_write(two.cache, k_want, v, *two.where)
    if not given:
        how["positions"] = None
    mark = torch.full((one.T, H, d), 7.0, dtype=BF16, device="cuda")
    q = s2a.s2a_rotate_write(one.cache, job.on_q, job.on_k, v, job.turns, *one.where, q_out=mark, **how)
    assert q is mark
    inside = one.rows()
    assert torch.equal(q[inside.cuda()], q_want[inside.cuda()]) and (q[~inside.cuda()] == 7).all()
    for x, y in zip(one.host_cache().values(), two.host_cache().values()):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert s2a.device_status() == (0, 0)


def test_bad_batches_are_reported_and_skipped():
    from test_gpu_paged import Job as CacheJob

    one = CacheJob([(3, 50), (2, 20)], Hkv=2, H=4, d=64, page=16)
    job = Job(one.T, 4, 2, 64)
    v = job.on_k.clone()
    before = one.host_cache()
    for bad, where in ((1003, (torch.full_like(one.table, one.cache.k.shape[0]), one.starts, one.lengths)), (1002, (one.table, one.starts, one.lengths * 0)),
                       (1001, (one.table, one.starts + 1, one.lengths))):
        s2a.s2a_rotate_write(one.cache, job.on_q, job.on_k, v, job.turns, *where)
        torch.cuda.synchronize()
        with pytest.raises(s2a.S2AError):
            s2a.s2a_rotate(job.on_q, job.on_k, job.turns)
        assert s2a.device_status() == (s2a.S2A_ERR_BAD_INDEX, bad) and s2a.device_status() == (0, 0)
        if bad == 1003:
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before.values(), one.host_cache().values()))


# ---------------------------------------------------------------------------------------------- autograd
@pytest.mark.parametrize("norm,weights", [(None, BF16), ("plain", BF16), ("weights", BF16), ("weights", F32)])
def test_autograd_gives_the_gradients_of_the_formula(norm, weights):
    job = Job(30, 4, 2, 64, norm=norm, weights=weights, packed=True)
    leaves = [t.detach().clone().requires_grad_() if t is not None else None for t in (job.on_q, job.on_k, *(None if w is None else w.cuda() for w in (job.qw, job.kw)))]
    q, k = s2_rotate(leaves[0], leaves[1], job.turns, job.positions.cuda(), q_weight=leaves[2], k_weight=leaves[3], eps=job.eps)
    want = s2a.s2a_rotate_bwd(job.on_q, job.on_k, job.dq_out.cuda(), job.dk_out.cuda(), job.turns, **job.how)
    given = [x for x in leaves if x is not None]
    got = torch.autograd.grad((q, k), given, (job.dq_out.cuda(), job.dk_out.cuda()), retain_graph=True)
    for g, w, x in zip(got, [w for w in want if w is not None], given):
        assert g.dtype == x.dtype and torch.equal(g, w.to(x.dtype))
    # one result alone: the other one's gradient is zero
    alone = torch.autograd.grad(k, given, job.dk_out.cuda())
    assert (alone[0] == 0).all() and torch.equal(alone[1], got[1])
    if norm == "weights":
        assert (alone[2] == 0).all() and torch.equal(alone[3], got[3])


def test_autograd_takes_strides_and_expanded_gradients():
    job = Job(24, 4, 2, 64, norm="weights")
    x = job.on_q.transpose(0, 1).contiguous().transpose(0, 1).requires_grad_()  # heads are not together
    q, k = s2_rotate(x, job.on_k, job.turns, eps=job.eps)
    q.sum().backward()
    want = s2a.s2a_rotate_bwd(job.on_q, job.on_k, torch.ones_like(job.on_q), torch.zeros_like(job.on_k), job.turns, eps=job.eps)
    assert torch.equal(x.grad, want[0])


def column(x, n):
    return torch.full((x.shape[0], n), 0.5, dtype=x.dtype, device=x.device)


# what comes back for the rotated queries is ..
LATER = [("the same for all tokens", lambda y: y.sum(0)), ("behind three columns more", lambda y: torch.cat((y.flatten(1), column(y, 3)), 1)),
         ("off 16 bytes", lambda y: torch.cat((column(y, 4), y.flatten(1)), 1)), ("the same for two tokens at a time", lambda y: y.view(-1, 2, *y.shape[1:]).sum(1)),
         ("off 16 bytes and dense", lambda y: torch.cat((column(y, 1)[0], y.flatten())))]


@pytest.mark.parametrize("later", [f for _, f in LATER], ids=[x for x, _ in LATER])
@pytest.mark.parametrize("norm", [None, "weights"])
def test_autograd_takes_gradients_as_they_come(later, norm):
    g = torch.Generator().manual_seed(3)
    job = Job(24, 4, 2, 64, norm=norm)
    leaves = [t.clone().requires_grad_() for t in (job.on_q, job.on_k)]
    q, k = s2_rotate(*leaves, job.turns, **job.how)
    y = q.detach().requires_grad_()
    out = later(y)
    gradient = numbers(g, *out.shape).cuda()
    dy, = torch.autograd.grad(out, y, gradient)
    got = torch.autograd.grad((later(q), k), leaves, (gradient, job.dk_out.cuda()))
    want = s2a.s2a_rotate_bwd(job.on_q, job.on_k, dy.clone(memory_format=torch.contiguous_format), job.dk_out.cuda(), job.turns, **job.how)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_autograd_takes_a_gradient_for_all_sequences_and_tokens():
    job = Job(24, 4, 2, 64)
    for B, axes in ((3, (0, 1)), (1, 1), (24, 0)):
        x = job.on_q.view(B, 24 // B, 4, 64).detach().requires_grad_()
        q, _ = s2_rotate(x, job.on_k.view(B, 24 // B, 2, 64), job.turns)
        (q.sum(axes) * job.dq_out[0].cuda()).sum().backward()
        dy = job.dq_out[:1].cuda().expand(24, 4, 64).contiguous().view_as(x)
        want = s2a.s2a_rotate_bwd(None, None, dy, torch.zeros_like(job.on_k).view(B, 24 // B, 2, 64), job.turns)
        assert torch.equal(x.grad, want[0])


@pytest.mark.parametrize("norm", [None, "weights"])
@pytest.mark.parametrize("kind", ["odd distance", "off 16 bytes", "one token for all", "rows that overlap", "far apart"])
def test_autograd_takes_tokens_at_any_distance(norm, kind):
    T, H, d = (2 if kind == "far apart" else 10), 4, 64
    job = Job(T, H, 2, d, norm=norm)
    stride, first = {"odd distance": (H * d + 3, 0), "off 16 bytes": (H * d + 8, 4), "one token for all": (0, 0), "rows that overlap": (64, 0), "far apart": (2**28 + 8, 0)}[kind]
    memory = torch.zeros((T - 1) * stride + H * d + first, dtype=BF16, device="cuda")
    memory[first:first + H * d * (2 if stride >= 64 else 1)].copy_(numbers(torch.Generator().manual_seed(2), 2 * H * d)[:H * d * (2 if stride >= 64 else 1)])
    x = memory.as_strided((T, H, d), (stride, d, 1), first).requires_grad_()
    copy = x.detach().clone(memory_format=torch.contiguous_format)
    got = s2_rotate(x, job.on_k, job.turns, **job.how)
    want = s2a.s2a_rotate(copy, job.on_k, job.turns, **job.how)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dx, = torch.autograd.grad(got, x, (job.dq_out.cuda(), job.dk_out.cuda()))
    assert torch.equal(dx, s2a.s2a_rotate_bwd(copy, job.on_k, job.dq_out.cuda(), job.dk_out.cuda(), job.turns, **job.how)[0])


@pytest.mark.parametrize("norm", [None, "plain", "weights"])
def test_second_derivatives_are_refused(norm):
    job = Job(24, 4, 2, 64, norm=norm)
    how = job.how
    leaves = [t.clone().requires_grad_() for t in (job.on_q, job.on_k)]
    if norm == "weights":
        leaves += [how["q_weight"].requires_grad_(), how["k_weight"].requires_grad_()]

    def first(create_graph):
        q, k = s2_rotate(*leaves[:2], job.turns, **how)
        return torch.autograd.grad(q.float().square().sum() + k.float().square().sum(), leaves, create_graph=create_graph)

    want, got = first(False), first(True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for leaf in leaves:
        with pytest.raises(NotImplementedError, match="second derivatives"):
            torch.autograd.grad(sum(x.float().sum() for x in got), leaf, retain_graph=True, allow_unused=True)
    # gradients that do not depend on anything are as ever
    q, _ = s2_rotate(*leaves[:2], job.turns, **how)
    dq, = torch.autograd.grad(q, leaves[0], job.dq_out.cuda(), create_graph=True)
    assert dq.requires_grad == (norm is not None)


def test_gradients_into_attention():
    """Rotated queries and keys in shifted sparse attention: the whole chain's gradients against finite parts computed in 64 bits."""
    g = torch.Generator().manual_seed(4)
    B, N, H, d, G = 1, 256, 2, 64, 128
    q, k, v, dO = (numbers(g, B, N, H, d) for _ in range(4))
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(BF16)
    from paper_2309_12307_b200.autograd import s2_attn

    turns = s2a.rotary_turns(d, scale=0.5)
    on = [t.cuda().requires_grad_() for t in (q, k, v, w)]
    a, b = s2_rotate(on[0], on[1], turns, q_weight=on[3], k_weight=on[3], eps=1e-5)
    s2_attn(a, b, on[2], G).backward(dO.cuda())
    full = [t.double().requires_grad_() for t in (q, k, v, w)]
    count, freq = torch.arange(N), torch.tensor(radians(d, scale=0.5), dtype=torch.float64)
    angle = count.double()[:, None] * freq

    def rot(x):
        x = x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * full[3]
        u, t = x[..., :d // 2], x[..., d // 2:]
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        return torch.cat((u * c - t * s, u * s + t * c), -1)

    half = H // 2

    def attend(x, y, z, shift):
        x, y, z = (t.roll(-shift, 1).reshape(N // G, G, -1, d).transpose(1, 2) for t in (x, y, z))
        score = (x @ y.transpose(-1, -2)) / math.sqrt(d)
        score = score.masked_fill(torch.ones(G, G, dtype=torch.bool).triu(1), -math.inf)
        return (score.softmax(-1) @ z).transpose(1, 2).reshape(1, N, -1, d).roll(shift, 1)

    x, y = rot(full[0]), rot(full[1])
    o = torch.cat([attend(x[:, :, s], y[:, :, s], full[2][:, :, s], shift) for s, shift in ((slice(0, half), 0), (slice(half, H), G // 2))], 2)
    o.backward(dO.double())
    # the parity tests' tolerance for gradients of attention; q and k are rounded once more on the way, and so are their gradients
    for got, want in zip(on, full):
        rel = float((got.grad.double().cpu() - want.grad).norm() / want.grad.norm())
        assert rel <= 1e-2, rel


def test_a_captured_step():
    """Forward and backward pass of a step in a CUDA graph."""
    job = Job(32, 4, 2, 64, norm="weights")
    q, k, w = job.on_q.requires_grad_(), job.on_k.requires_grad_(), job.qw.cuda().requires_grad_()
    positions = job.positions.cuda()
    dq, dk = job.dq_out.cuda(), job.dk_out.cuda()

    def step():
        out = s2_rotate(q, k, job.turns, positions, q_weight=w, k_weight=w, eps=1e-5)
        return torch.autograd.grad(out, (q, k, w), (dq, dk))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        dq.neg_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


# ---------------------------------------------------------------------------------------------- refusals
def test_refusals():
    job = Job(8, 4, 2, 64, norm="weights")
    q, k, t = job.on_q, job.on_k, job.turns
    w = job.qw.cuda()
    for message, call in [("q must have dtype", lambda: s2a.s2a_rotate(q.float(), k, t)), ("k must have dtype", lambda: s2a.s2a_rotate(q, k.half(), t)),
                          ("k must be a CUDA", lambda: s2a.s2a_rotate(q, k.cpu(), t)), ("k must be", lambda: s2a.s2a_rotate(q, k[:4], t)),
                          ("q must have dense heads", lambda: s2a.s2a_rotate(q[:, ::2], k, t)), ("turns must have dtype", lambda: s2a.s2a_rotate(q, k, t.int())),
                          ("turns must be", lambda: s2a.s2a_rotate(q, k, t.repeat(2))), ("positions must have dtype", lambda: s2a.s2a_rotate(q, k, t, t)),
                          ("positions must be one", lambda: s2a.s2a_rotate(q, k, t, t[:5].int())), ("belong to a norm", lambda: s2a.s2a_rotate(q, k, t, q_weight=w)),
                          ("q_weight must have dtype", lambda: s2a.s2a_rotate(q, k, t, q_weight=w.half(), eps=0.0)),
                          ("k_weight must have dtype", lambda: s2a.s2a_rotate(q, k, t, q_weight=w, k_weight=w.float(), eps=0.0)),
                          ("k_weight must have shape", lambda: s2a.s2a_rotate(q, k, t, k_weight=w[:32], eps=0.0)),
                          ("q_out must have shape", lambda: s2a.s2a_rotate(q, k, t, q_out=k)), ("q must be a torch.Tensor", lambda: s2a.s2a_rotate(None, k, t)),
                          ("dk_out must be", lambda: s2a.s2a_rotate_bwd(q, k, q, q[:4], t)), ("q must have shape", lambda: s2a.s2a_rotate_bwd(k, k, q, k, t, eps=0.0)),
                          ("q must have dtype", lambda: s2_rotate(q.float(), k, t)), ("q must be a torch.Tensor", lambda: s2_rotate(3, k, t))]:
        with pytest.raises(ValueError, match=message):
            call()
    for status, call in [(s2a.S2A_ERR_UNSUPPORTED, lambda: s2a.s2a_rotate(q, k, t[:4])), (s2a.S2A_ERR_INVALID_ARG, lambda: s2a.s2a_rotate(q, k, t, eps=-1.0)),
                         (s2a.S2A_ERR_INVALID_ARG, lambda: s2a.s2a_rotate(q, k, t, eps=math.nan)),
                         (s2a.S2A_ERR_INVALID_ARG, lambda: s2a.s2a_rotate(q[:1].expand(8, 4, 64), k, t)),
                         (s2a.S2A_ERR_UNSUPPORTED, lambda: s2a.s2a_rotate(q[..., :32].contiguous(), k[..., :32].contiguous(), t[:16])),
                         (s2a.S2A_ERR_UNSUPPORTED, lambda: s2_rotate(q, k, t[:4]))]:
        with pytest.raises(s2a.S2AError) as e:
            call()
        assert e.value.status == status
    assert s2a.device_status() == (0, 0)
