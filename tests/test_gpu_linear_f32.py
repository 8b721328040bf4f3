"""The product in float32: errors of float32 on the tensor cores too (operands in three bf16 parts, six of the nine products)."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def kernels(f):
    """Names of the library's kernels that f launches; none where the profiler sees no kernels."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA], acc_events=True) as prof:
        f()
        torch.cuda.synchronize()
    return [e.key for e in prof.key_averages() if "dare::" in e.key]


# k-elements that are no multiple of a block of 64, shared by clusters of 2, 4 and 8 CTAs of unequal numbers of blocks, or by none; the launch
# rule is clear about each (the form it takes is estimated at 0.9 of the other's time and less).
TENSOR = [(20, 2052, 2048), (40, 4164, 1500), (128, 2052, 2048), (300, 4164, 1024), (200, 1036, 3001), (77, 8196, 1000), (33, 2052, 2047),
          (48, 16388, 448), (601, 1028, 1000), (5000, 136, 512), (2000, 132, 515), (250, 1156, 1999), (640, 1024, 960)]
CORES = [(1, 4096, 600), (4, 1001, 333), (17, 2052, 500), (33, 516, 65), (90, 200, 64), (200, 129, 65), (50, 1001, 1000), (300, 2051, 400)]


@pytest.mark.parametrize("m,k,n,tensor", [(*s, True) for s in TENSOR] + [(*s, False) for s in CORES])
def test_errors_of_float32(dare, m, k, n, tensor):
    g = torch.Generator(device="cuda").manual_seed(m + k + n)
    x = torch.randn((m, k), generator=g, device="cuda")
    w = torch.randn((n, k), generator=g, device="cuda") * k ** -0.5
    y = dare.linear(x, w)
    err = y.double() - x.double() @ w.double().T
    size = (x.double().square() @ w.double().square().T).sqrt()
    # Errors (2-norms) in units of 2^-24 of sqrt(sum (x w)^2), what such a sum of k products of random signs is.
    # CUDA cores: at most k / 4 additions in a row (two groups, even and odd elements), each off by at most half a unit of a partial sum that
    # has grown like the square root of its terms: 0.3 sqrt(k / 4) if errors are spread evenly, 0.7 sqrt(k / 4) if all were largest;
    # the sums of the parts, 3.
    # Tensor cores: what three parts leave, 0.5; products of scale 2^-8 summed by truncating additions, k / 16 of them, a unit of 2^-23 of
    # 2^-8 of the sum each, in three accumulators: k / 680; chains of at most max(4, k / 512) rounded additions, the rest of the tree and
    # the last sums: below 5.  One of the six products left out: 40 and more; one part: 39000.
    bound = 6 + k / 680 if tensor else 3 + 0.7 * (k / 4) ** 0.5
    got = err.norm().item() / size.norm().item() * 2 ** 24
    assert got <= bound < 35, (got, bound)
    # No element far out: its error is a sum of many independent ones; eight times the bound on their 2-norm.
    assert bool((err.abs() <= 8 * bound * 2.0 ** -24 * size).all())
    names = kernels(lambda: dare.linear(x, w))
    assert not names or any("gemm_f32_kernel" in name for name in names) == tensor, names
    # the same rows and columns, whatever stands beside them
    assert torch.equal(dare.linear(x, w), y)
    print("%d x %d x %d %s: %.2f of %.1f" % (m, k, n, "tensor" if tensor else "cores", got, bound))


@pytest.mark.parametrize("m,k,n", [(40, 4164, 1500), (300, 4164, 1024), (77, 8196, 1000), (48, 16388, 448)])
def test_not_numbers_in_the_last_part(dare, m, k, n):
    """In the last of a cluster's parts, whose block of k-elements is filled up with zeros: its row and its column, nothing else."""
    g = torch.Generator(device="cuda").manual_seed(n)
    x, w = torch.randn((m, k), generator=g, device="cuda"), torch.randn((n, k), generator=g, device="cuda")
    plain = dare.linear(x, w)
    x[m - 1, k - 1], w[n - 1, k - 2] = float("inf"), float("nan")
    got = dare.linear(x, w)
    assert torch.equal(got[:m - 1, :n - 1], plain[:m - 1, :n - 1])
    assert bool(got[:, n - 1].isnan().all()) and bool(got[m - 1, :n - 1].isinf().all())
    assert torch.equal(got[m - 1, :n - 1].sign(), w[:n - 1, k - 1].sign())


@pytest.mark.parametrize("m,k,n", [(1, 4, 3001), (4, 64, 1000), (30, 64, 500), (1000, 512, 640)])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activations_keep_small_results(dare, act, m, k, n):
    """Where an activation is nearly zero it is still right in relation to its value: arguments one after the other, products with one."""
    v = torch.linspace(-9, 9, m * n, device="cuda").view(m, n)
    if m > 4:
        v = v[:, :1].expand(m, n)                            # (an argument a row)
    x, w = torch.zeros((m, k), device="cuda"), torch.zeros((n, k), device="cuda")
    # (the products are exact: one factor is 1, or for few rows a power of two)
    if m > 4:
        x[:, 0], w[:, 0] = v[:, 0], 1
        arg = v.double()
    else:
        x[:, 0], w[:, 0] = 2.0 ** torch.arange(0, -m, -1, device="cuda"), v[0]
        arg = x[:, :1].double() * w[:, 0].double()
    got = dare.linear(x, w, act=dare.ACT[act]).double()
    if act == "silu":
        want, slope = arg / (1 + (-arg).exp()), arg.abs()
    elif act == "gelu":
        want, slope = 0.5 * arg * torch.special.erfc(-arg / 2 ** 0.5), arg.square()
    else:
        u = (2 / torch.pi) ** 0.5 * (arg + 0.044715 * arg ** 3)
        want, slope = arg / (1 + (-2 * u).exp()), 8 * u.abs()
    # A function of a rounded argument z (half a unit, for tanh's polynomial in z four units) is off by z times its logarithm's slope of
    # them; the functions themselves and the operations around them by at most eight units of 2^-23.
    assert bool(((got - want).abs() <= (8 + slope) * 2.0 ** -23 * want.abs()).all()), ((got - want).abs() / want.abs().clamp(min=1e-300)).max().item()
