"""Host-side rules of the calls for many prompts (no GPU needed): refusals before anything is launched, workspace sizes."""
import itertools

from paper_2604_09244_amd import binding as mv


def test_null_arguments_are_refused():
    lib = mv.load()
    assert lib.mvla_rotation_table(None, None, 1, None, None) == -1
    assert lib.mvla_rotate(None, None, 1, None, None, 0, None, None, 1, 1, 64, 64, 0, 0, None, None, 1) == -1
    assert lib.mvla_pages_append(None, None, None, None, None, 1) == -1
    assert lib.mvla_pages_read(None, None, None, None, 1, None, None) == -1
    assert lib.mvla_pages_attention(None, None, None, None, 1, 1, 1, 1, 1.0, None, None) == -1
    assert lib.mvla_logprobs(None, None, 0, 1, 1, 1, None, None, 0, None, None, 0, None, None) == -1


def test_workspace_sizes():
    f = mv.load().mvla_pages_workspace_bytes
    good = (4, 32, 8, 128, 600, 512, 4096)
    assert f(*good) > 0
    for i, bad in ((0, 0), (1, 0), (1, 30), (2, 0), (3, 96), (4, 0), (5, 0), (6, 0), (0, 70000), (4, 2 ** 28), (6, 2 ** 31 - 1), (2, -8)):
        args = list(good)
        args[i] = bad
        assert f(*args) == 0, args
    # grows with every argument, so that a context made for the largest call takes every smaller one
    steps = [(1, 3, 64), (4, 16, 32), (1, 40, 700), (1, 4, 5, 16, 17, 300), (1, 33, 5000)]
    for B, H, n, q, length in itertools.product(*steps):
        here = f(B, H, 4, 128, n, q, length)
        for i, s in enumerate(steps):
            v = (B, H, n, q, length)[i]
            if v != s[-1]:
                up = [B, H, n, q, length]
                up[i] = s[s.index(v) + 1]
                assert f(up[0], up[1], 4, 128, *up[2:]) >= here, (B, H, n, q, length, i)
    assert f(*good) >= mv.load().mvla_cache_workspace_bytes(1, 1, 1, 64, 1, 32) // 2


def test_names_of_the_kernels():
    lib = mv.load()
    assert [lib.mvla_kernel_name(i).decode() for i in range(23, 30)] == ["sample", "rotate", "pages_append", "pages_read",
                                                                         "pages_attention", "logprobs", "?"]
