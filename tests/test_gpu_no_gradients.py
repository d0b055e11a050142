"""The operators on 4-bit codes have no gradients: tensors that want them are refused rather than cut off without a word."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def calls():
    """Each call as (function, arguments, names of the arguments that may want gradients)."""
    import paper_2608_18147_gb300 as E
    x = torch.randn(2, 128, device="cuda")
    idx = torch.randint(0, 16, (32, 128), dtype=torch.uint8, device="cuda")
    product = dict(x=x, codes=E.ecasq_pack(idx), levels=torch.randn(16, device="cuda"), scales=torch.rand(32, 4, device="cuda"), group=32)
    rows = torch.randn(2, 16, 1, 32, device="cuda")
    plain = dict(q=torch.randn(1, 2, 32, device="cuda"), k=rows, v=rows.clone(), table=torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"),
                 lengths=torch.tensor([20], dtype=torch.int32, device="cuda"))
    codes = torch.randint(0, 100, (2, 16, 1, 16), dtype=torch.uint8, device="cuda")
    levels = torch.randn(2, 16, 1, 8, device="cuda").half()
    coded = dict(plain, q=plain["q"].half(), k=codes, v=codes, k_levels=levels, v_levels=levels.clone())
    write = dict(x=torch.randn(3, 1, 32, device="cuda"), Q=torch.randn(3, 8, device="cuda").sort(dim=1).values, m=None,
                 slots=torch.arange(3, device="cuda"), codes=codes.clone(), levels=levels.clone(), seed=1)
    return [(E.ecasq_matvec, product, ("x", "levels", "scales")), (E.ecasq_attend, plain, ("q", "k", "v")),
            (E.ecasq_attend, coded, ("q", "k_levels", "v_levels")), (E.ecasq_cache_write, write, ("x", "Q", "levels"))]


def test_inputs_that_require_gradients_are_refused():
    import paper_2608_18147_gb300 as E
    for fn, args, names in calls():
        fn(**args)
        for name in names:
            wants = dict(args, **{name: args[name].clone().requires_grad_()})
            with pytest.raises(E.EcasqError, match="gradient"):
                fn(**wants)
            with torch.no_grad():
                fn(**wants)
            with torch.inference_mode():
                fn(**wants)
            fn(**dict(args, **{name: wants[name].detach()}))


def test_outputs_that_require_gradients_are_refused():
    import paper_2608_18147_gb300 as E
    (product, args, _), (attend, plain, _) = calls()[:2]
    for fn, a, like in ((product, args, torch.empty(2, 32, device="cuda")), (attend, plain, torch.empty_like(plain["q"]))):
        with pytest.raises(E.EcasqError, match="gradient"):
            fn(**a, out=like.clone().requires_grad_())
        fn(**a, out=like)


def test_dual_tensors_are_refused():
    import torch.autograd.forward_ad as ad
    import paper_2608_18147_gb300 as E
    for fn, args, names in calls():
        with ad.dual_level():
            fn(**args)
            for name in names:
                dual = ad.make_dual(args[name], torch.ones_like(args[name]))
                with pytest.raises(E.EcasqError, match="gradient"):
                    fn(**dict(args, **{name: dual}))
