"""The head's answers, orthogonalised steps and 8-bit weights where offsets pass 32 bits, values and bytes, against the definitions in 64 bits."""
import pytest
import torch

import paper_1502_03409_amd as lc
import test_gpu_logp as logp
import test_gpu_muon as muon
import test_gpu_q8 as q8

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]


def ids(dtype):
    return "bf16" if dtype == torch.bfloat16 else "f32"


def normal(shape, dtype, std, seed):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0, std, generator=torch.Generator("cuda").manual_seed(seed))


@pytest.mark.parametrize("N", [3, 40, 300])       # few rows, a mini-batch, tiles
def test_a_vocabulary_of_more_than_2_31_values(N):
    V, D, T, K = 600000, 4096, 2, 5
    print(f"case logp {N} x {D} over {V} words", flush=True)
    x, w = normal((N, D), torch.bfloat16, 1.0, 0), normal((V, D), torch.bfloat16, 2 * D ** -0.5, 1)
    tags = torch.randint(0, V, (N, T), generator=torch.Generator().manual_seed(2)).cuda()
    tags[0, 0], tags[N - 1, 1], tags[1] = V - 1, V - 2, -1
    got = logp.answers(x, w, tags, K)
    want = logp.definition(x, w, tags, K)
    b = logp.check_answers(x, w, tags, K, got, want)
    dlogp, dentropy = logp.upstream(N, T)
    dlogp = torch.where(tags >= 0, dlogp, 0.0)
    dentropy = torch.where(want["live"], dentropy, 0.0)
    grads = logp.gradients(x, w, tags, got, dlogp, dentropy)
    logp.check_gradients(x, w, tags, dlogp, dentropy, grads, b, want)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_weights_of_more_than_2_32_bytes_in_8_bits(dtype):
    F, D, ends = 1 << 20, 4200, 3000
    print(f"case q8 {D} -> {F} {dtype}", flush=True)
    w = normal((F, D), dtype, D ** -0.5, 3)
    q, s = q8.rows(w)
    assert q.numel() > 1 << 32
    parts = [slice(0, ends), slice(F // 2 - ends, F // 2 + ends), slice(F - ends, F)]
    for p in parts:
        want, scale = q8.q8(w[p])
        assert torch.equal(s[p], scale) and torch.equal(q[p][:, :D].double(), want) and not q[p][:, D:].any()
    qu, su = q.roll(-ends, 0), s.roll(-ends)
    for N in (2, 150, 300):
        x = normal((N, D), dtype, 1.0, 4 + N)
        y, h = q8.matmul(x, q, s), q8.glu(x, q, s, qu, su, "sigmoid")
        for p in parts:
            g = q8.want_matmul(x, w[p])
            q8.close(y[:, p], g)
            u = q8.want_matmul(x, torch.cat([w[p.start + ends:p.stop + ends], w[:max(0, p.stop + ends - F)]]))
            want = torch.sigmoid(g) * u
            # both sums rounded to fp32 and scaled twice, a sigmoid (whose slope is at most a quarter of itself times |g|), a product, the result's rounding
            step = (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) + 2.0 ** -21
            assert ((h[:, p].double() - want).abs() <= step * (1 + g.abs()) * want.abs() + 2.0 ** -100).all()


@pytest.mark.parametrize("dtype,shape", [(torch.bfloat16, (9000, 512, 512)), (torch.float32, (40, 1 << 20, 60)), (torch.bfloat16, (300, 100, 80000))], ids=str)
def test_stacks_of_more_than_2_31_values(dtype, shape):
    print(f"case muon {shape} {dtype}", flush=True)
    w, g, m = normal(shape, dtype, 0.5, 5), normal(shape, dtype, 1.0, 6), normal(shape, torch.float32, 4.0, 7)
    assert w.numel() > 1 << 31
    n = shape[0]
    at = [0, n // 2, n - 1]
    old = [t[at].clone() for t in (w, g, m)]
    lc.muon_step(w, g, m, None, None, 0.3, 0.01, 0.9, True, 5, muon.code(dtype), muon.scratch(shape, dtype))
    muon.check((w[at], m[at]), *old, bounds=True)


def test_the_most_rows_and_matrices():
    """2^24, of one value each: more workgroups of 256 threads than a launch takes."""
    N = 1 << 24
    x, w = normal((N, 1), torch.float32, 1.0, 8), normal((2, 1), torch.float32, 1.0, 9)
    q, s = q8.rows(x)
    assert torch.equal(s, (x.abs()[:, 0] / torch.full_like(s, 127)).clamp(min=2.0 ** -126))
    assert torch.equal(q[:, 0].float(), 127 * torch.sign(x[:, 0])) and not q[:, 1:].any()
    del q, s
    tags = torch.arange(N, device="cuda")[:, None] % 3 - 1
    got, want = logp.answers(x, w, tags, 1), logp.definition(x, w, tags, 1)
    b = logp.check_answers(x, w, tags, 1, got, want)
    dlogp, dentropy = normal((N, 1), torch.float32, 1.0, 10), normal((N,), torch.float32, 1.0, 11)
    dx = logp.gradients(x, w, tags, got, dlogp, dentropy)[0].double()
    d = logp.d_of(want, tags, dlogp, dentropy) @ w.double()
    assert float((dx - d).norm()) <= 8 * b * float(d.norm())
    del got, want, d, dx
    u, g, m = torch.zeros(N, 1, 1, device="cuda"), x[:, :, None].contiguous(), torch.zeros(N, 1, 1, device="cuda")
    lc.muon_step(u, g, m, None, None, 1.0, 0.0, 0.9, True, 1, lc.LC_F32, muon.scratch((N, 1, 1), torch.float32))
    assert torch.equal(m, g)
    one = muon.A + muon.B + muon.C       # a matrix of one value becomes its sign
    # three products of values with 22 bits, each at most 4.8, one on the way to S and two to P X
    assert ((u[:, 0, 0].double() + one * torch.sign(x[:, 0])).abs() <= 6 * 4.8 * 2.0 ** -22).all()
