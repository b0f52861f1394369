"""One test for many combinations: what a test of its own costs each (the allocator's memory handed back, garbage collected) is more than the cases themselves."""
import inspect
import itertools


def every(**sets):
    """Runs the test with each combination of these arguments' values, which it names when one fails."""
    def wrap(test):
        def run(**given):
            for values in itertools.product(*sets.values()):
                case = dict(zip(sets, values))
                print(test.__name__, given, case, flush=True)
                try:
                    test(**given, **case)
                except AssertionError as e:
                    raise AssertionError(case) from e
        run.__name__, run.__doc__, run.__module__ = test.__name__, test.__doc__, test.__module__
        run.one = test
        own = inspect.signature(test)
        run.__signature__ = own.replace(parameters=[p for n, p in own.parameters.items() if n not in sets])
        return run
    return wrap
