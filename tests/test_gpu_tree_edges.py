"""Calls of the tree operators that the documentation allows and that lie at its edges."""
import threading

import pytest
import torch

import tree_ref as tree

pytestmark = pytest.mark.gpu

siso = pytest.importorskip("paper_2508_18736_b200")
I32 = dict(dtype=torch.int32, device="cuda")


def test_verifications_of_two_threads_with_different_vocabularies():
    # how much shared memory a kernel may have belongs to the kernel, not to the call: what one thread asks for must not be taken from another's launch
    wrong = []

    def work(vocab, seed):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                g = torch.Generator(device="cuda").manual_seed(seed)
                target = torch.softmax(torch.randn((3, vocab), device="cuda", generator=g), -1)
                tokens, parents, cu = (torch.tensor(x, **I32) for x in ([0, 5, 7], [-1, 0, 0], [0, 3]))
                u, us = torch.rand(3, device="cuda", generator=g), torch.rand(1, device="cuda", generator=g)
                want = tree.verify_tree(target, None, tokens, parents, [0, 3], 2, u, us)
                for _ in range(3000):
                    got = siso.verify_tree(target, None, tokens, parents, cu, 2, u, us)
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a.cpu(), b) for a, b in zip(got, want)):
                    wrong.append("tokens differ")
        except Exception as e:
            wrong.append(str(e))

    threads = [threading.Thread(target=work, args=a) for a in ((262144, 1), (60000, 2), (131072, 3), (50000, 4))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
