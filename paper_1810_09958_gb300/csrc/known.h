// known.h -- answers of a query that costs host time, kept under a key.
#pragma once
#include <mutex>

namespace isam {

// A query that fails gives no answer: its status goes to the caller, and the
// next call asks again.  Key needs ==; beyond CAP keys nothing more is kept.
template <typename Key, int CAP>
class Known {
public:
    // ask(n) fills in *n and returns 0, or a status.
    template <typename Ask>
    int get(const Key &key, int *n, Ask &&ask) {
        std::lock_guard<std::mutex> lk(mu_);
        for (int i = 0; i < count_; ++i)
            if (kept_[i].key == key) {
                *n = kept_[i].n;
                return 0;
            }
        const int rc = ask(n);
        if (rc == 0 && count_ < CAP) kept_[count_++] = {key, *n};
        return rc;
    }

private:
    struct Entry {
        Key key;
        int n;
    };
    std::mutex mu_;
    Entry kept_[CAP];
    int count_ = 0;
};

}  // namespace isam
